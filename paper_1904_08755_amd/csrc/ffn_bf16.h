// Tile product of bfloat16 operands for the feed-forward block (ffn.hip): the operands go from
// memory straight into LDS, in a ring of three stages of 32 reduction elements.
//
// A step waits until its own stage has landed (the next one stays in flight), passes one barrier, starts the
// copies of the step after next into the stage that the step before has read, reads its fragments
// and multiplies.  Copies are buffer loads that write 1 KiB of LDS (64 lanes x 16 bytes) and read zeros
// outside the operand, so odd ends need no other code; they take 16-byte pieces, so operands' rows
// must be whole pieces at 16-byte addresses.
//
// Layouts of a stage (a load writes lane after lane, so the permutation is applied to the piece each lane fetches):
//   KC, the reduction along the rows: rows of 64 bytes, piece c of row r at (c ^ ((r >> 1) & 3)) * 16, for
//       operands of 32 rows at (c ^ ((r >> 2) & 3)) * 16; fragments are 16-byte reads.
//   MC, the reduction across the rows: a line of 64, 128 or 256 columns per reduction element k, its 32-byte
//       pairs of pieces permuted by bits of k such that the eight lines which a transpose read
//       (ds_read_b64_tr_b16) serves together lie in distinct banks; of an operand in blocks (row_blocks) lines
//       of 32 columns, 32 of them after each other, so that a load takes 1 KiB of a block.  Within each 16 lanes, lane i of such a
//       read receives element i % 4 of the 8-byte pieces that lanes i / 4, i / 4 + 4, ... address.
//
// A step's LDS reads are one block of inline assembly that also waits for them: the compiler cannot tell
// which stage a read touches and would wait for every copy in flight before each.
#pragma once

#include "row_vec.h"

namespace gsc {

typedef __bf16 fbf16x8 __attribute__((ext_vector_type(8)));
typedef short fs16x4 __attribute__((ext_vector_type(4)));

constexpr int kFbStages = 3;

// s_waitcnt operand: vmcnt(n), the other counters left free (gfx9 encoding)
template <int N>
__device__ __forceinline__ void fb_wait() {
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | (7 << 4) | (15 << 8));
}
__device__ __forceinline__ void fb_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

// One side of a product: element (r, k) at row r and column k of m (KC), or row k and column r (MC), r < rows, k < the
// product's reduction length (both whole pieces along m's rows).
struct FbSide {
    RowMat<const uint16_t> m;
    int64_t rows;
};

// How a side lies: the reduction along its rows, across them, or across them in blocks.
enum FbLay { FB_KC, FB_MC, FB_MB };

// The copies of R rows (columns) of a side by a block of NW waves.
// T32: KC operands of 32 x 32 tiles.
template <FbLay LAY, int R, int NW, bool T32 = false>
struct FbCopy {
    static constexpr int INS = R / 16;                        // load instructions (1 KiB) of a stage
    static constexpr int N = (INS + NW - 1) / NW;             // ... per wave
    static constexpr int BYTES = R * 64;
    static constexpr int LINE = LAY == FB_MB ? 64 : R * 2;    // MC, MB: bytes of a line
    static constexpr int LPI = 1024 / LINE;                   // ... lines of an instruction (R <= 512)
    static constexpr int HALF = 4 * LINE;                     // ... four lines on: the second half of a transpose read
    static_assert(INS % NW == 0, "waves share a stage's copies evenly");

    // permutation of a line's pairs
    static __device__ __forceinline__ int perm(int k) {
        if (LAY == FB_MB) return (k >> 3) & 1;
        return R == 64 ? ((k >> 1) & 1) | ((k >> 2) & 2) : (k & 3) | ((k >> 1) & 4);
    }

    uint32_t off[N];   // byte offset of the lane's piece from the side's first element of the step
    int first[N];      // its first reduction element (relative to the step)

    __device__ __forceinline__ void start(const FbSide& s, int wave) {
        const int lane = threadIdx.x & 63;
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const int ins = wave * N + j;
            int row, col;   // of m; its piece's first column
            bool in;
            if (LAY == FB_KC) {
                row = ins * 16 + (lane >> 2);
                col = ((lane & 3) ^ ((lane >> (T32 ? 4 : 3)) & 3)) * 8;
                first[j] = col;
                in = row < s.rows;
            } else {
                row = (LAY == FB_MB ? ins % 2 : ins) * LPI + lane / (64 / LPI);
                const int slot = lane % (64 / LPI);
                col = ((((slot >> 1) ^ perm(row)) << 1) | (slot & 1)) * 8 + (LAY == FB_MB ? ins / 2 * 32 : 0);
                first[j] = row;
                in = col < s.rows;
            }
            off[j] = in ? (uint32_t)((row >> 7) * s.m.ts + (row & 127) * s.m.ld + (col >> 5) * s.m.gs + (col & 31)) * 2 : kBufNone;
        }
    }
    // the step at reduction element k0 of K, into LDS at dst
    __device__ __forceinline__ void issue(const FbSide& s, int64_t k0, int64_t K, uint8_t* dst, int wave) const {
        const uint16_t* base = LAY == FB_KC ? s.m.at(0, k0).p : s.m.at(k0, 0).p;
        // an upper bound of the bytes from there on that may be read; what lies outside the operand is masked below
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, 0x7fffffff, kBufFlags);
        const int left = (int)(K - k0 < 32 ? K - k0 : 32);   // (none from K on)
#pragma unroll
        for (int j = 0; j < N; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(dst + (wave * N + j) * 1024), 16,
                first[j] < left ? off[j] : kBufNone, 0, 0, 0);
    }
};

#define FB_R(o, a, off) "ds_read_b128 %" #o ", %" #a " offset:" #off "\n"
#define FB_T(o, a, off) "ds_read_b64_tr_b16 %" #o ", %" #a " offset:" off "\n"
#define FB_WAIT "s_waitcnt lgkmcnt(0)"

__device__ __forceinline__ fbf16x8 fb_join(fs16x4 lo, fs16x4 hi) {
    const fs16x4 v[2] = {lo, hi};
    return __builtin_bit_cast(fbf16x8, v);
}

// Four or eight KC blocks of A at a (1 KiB apart) with two or four KC blocks of B at b.
__device__ __forceinline__ void fb_read_kk(uint32_t a, uint32_t b, fbf16x8 (&A)[4], fbf16x8 (&B)[2]) {
    asm volatile(FB_R(4, 7, 0) FB_R(5, 7, 1024) FB_R(0, 6, 0) FB_R(1, 6, 1024) FB_R(2, 6, 2048) FB_R(3, 6, 3 * 1024) FB_WAIT
                 : "=&v"(A[0]), "=&v"(A[1]), "=&v"(A[2]), "=&v"(A[3]), "=&v"(B[0]), "=&v"(B[1])
                 : "v"(a), "v"(b)
                 : "memory");
}
__device__ __forceinline__ void fb_read_kk(uint32_t a, uint32_t b, fbf16x8 (&A)[4], fbf16x8 (&B)[4]) {
    asm volatile(FB_R(4, 9, 0) FB_R(5, 9, 1024) FB_R(6, 9, 2048) FB_R(7, 9, 3 * 1024) FB_R(0, 8, 0) FB_R(1, 8, 1024)
                     FB_R(2, 8, 2048) FB_R(3, 8, 3 * 1024) FB_WAIT
                 : "=&v"(A[0]), "=&v"(A[1]), "=&v"(A[2]), "=&v"(A[3]), "=&v"(B[0]), "=&v"(B[1]), "=&v"(B[2]), "=&v"(B[3])
                 : "v"(a), "v"(b)
                 : "memory");
}
__device__ __forceinline__ void fb_read_kk(uint32_t a, uint32_t b, fbf16x8 (&A)[8], fbf16x8 (&B)[4]) {
    asm volatile(FB_R(8, 13, 0) FB_R(9, 13, 1024) FB_R(10, 13, 2048) FB_R(11, 13, 3 * 1024) FB_R(0, 12, 0) FB_R(1, 12, 1024)
                     FB_R(2, 12, 2048) FB_R(3, 12, 3 * 1024) FB_R(4, 12, 4096) FB_R(5, 12, 5120) FB_R(6, 12, 6144)
                         FB_R(7, 12, 7168) FB_WAIT
                 : "=&v"(A[0]), "=&v"(A[1]), "=&v"(A[2]), "=&v"(A[3]), "=&v"(A[4]), "=&v"(A[5]), "=&v"(A[6]),
                   "=&v"(A[7]), "=&v"(B[0]), "=&v"(B[1]), "=&v"(B[2]), "=&v"(B[3])
                 : "v"(a), "v"(b)
                 : "memory");
}
// ... with four MC blocks of B at b[0..3], their second halves STEP bytes on.
template <int STEP>
__device__ __forceinline__ void fb_read_km(uint32_t a, const uint32_t (&b)[4], fbf16x8 (&A)[4], fbf16x8 (&B)[4]) {
    fs16x4 r[8];
    asm volatile(FB_T(4, 13, "0") FB_T(5, 13, "%17") FB_T(6, 14, "0") FB_T(7, 14, "%17") FB_T(8, 15, "0")
                     FB_T(9, 15, "%17") FB_T(10, 16, "0") FB_T(11, 16, "%17") FB_R(0, 12, 0) FB_R(1, 12, 1024)
                         FB_R(2, 12, 2048) FB_R(3, 12, 3 * 1024) FB_WAIT
                 : "=&v"(A[0]), "=&v"(A[1]), "=&v"(A[2]), "=&v"(A[3]), "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]),
                   "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]), "=&v"(r[7])
                 : "v"(a), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(STEP)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) B[i] = fb_join(r[2 * i], r[2 * i + 1]);
}
template <int STEP>
__device__ __forceinline__ void fb_read_km(uint32_t a, const uint32_t (&b)[4], fbf16x8 (&A)[8], fbf16x8 (&B)[4]) {
    fs16x4 r[8];
    asm volatile(FB_T(8, 17, "0") FB_T(9, 17, "%21") FB_T(10, 18, "0") FB_T(11, 18, "%21") FB_T(12, 19, "0")
                     FB_T(13, 19, "%21") FB_T(14, 20, "0") FB_T(15, 20, "%21") FB_R(0, 16, 0) FB_R(1, 16, 1024)
                         FB_R(2, 16, 2048) FB_R(3, 16, 3 * 1024) FB_R(4, 16, 4096) FB_R(5, 16, 5120) FB_R(6, 16, 6144)
                             FB_R(7, 16, 7168) FB_WAIT
                 : "=&v"(A[0]), "=&v"(A[1]), "=&v"(A[2]), "=&v"(A[3]), "=&v"(A[4]), "=&v"(A[5]), "=&v"(A[6]),
                   "=&v"(A[7]), "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]),
                   "=&v"(r[6]), "=&v"(r[7])
                 : "v"(a), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(STEP)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) B[i] = fb_join(r[2 * i], r[2 * i + 1]);
}
// Four MC blocks of each side.
template <int SA, int SB>
__device__ __forceinline__ void fb_read_mm(const uint32_t (&a)[4], const uint32_t (&b)[4], fbf16x8 (&A)[4], fbf16x8 (&B)[4]) {
    fs16x4 r[16];
    asm volatile(FB_T(8, 20, "0") FB_T(9, 20, "%25") FB_T(10, 21, "0") FB_T(11, 21, "%25") FB_T(12, 22, "0")
                     FB_T(13, 22, "%25") FB_T(14, 23, "0") FB_T(15, 23, "%25") FB_T(0, 16, "0") FB_T(1, 16, "%24")
                         FB_T(2, 17, "0") FB_T(3, 17, "%24") FB_T(4, 18, "0") FB_T(5, 18, "%24") FB_T(6, 19, "0")
                             FB_T(7, 19, "%24") FB_WAIT
                 : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]),
                   "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]),
                   "=&v"(r[14]), "=&v"(r[15])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(b[0]), "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(SA), "n"(SB)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        A[i] = fb_join(r[2 * i], r[2 * i + 1]);
        B[i] = fb_join(r[8 + 2 * i], r[9 + 2 * i]);
    }
}
template <int SA, int SB>
__device__ __forceinline__ void fb_read_mm(const uint32_t (&a)[8], const uint32_t (&b)[4], fbf16x8 (&A)[8], fbf16x8 (&B)[4]) {
    fs16x4 r[24];
    asm volatile(FB_T(16, 32, "0") FB_T(17, 32, "%37") FB_T(18, 33, "0") FB_T(19, 33, "%37") FB_T(20, 34, "0")
                     FB_T(21, 34, "%37") FB_T(22, 35, "0") FB_T(23, 35, "%37") FB_T(0, 24, "0") FB_T(1, 24, "%36")
                         FB_T(2, 25, "0") FB_T(3, 25, "%36") FB_T(4, 26, "0") FB_T(5, 26, "%36") FB_T(6, 27, "0")
                             FB_T(7, 27, "%36") FB_T(8, 28, "0") FB_T(9, 28, "%36") FB_T(10, 29, "0") FB_T(11, 29, "%36")
                                 FB_T(12, 30, "0") FB_T(13, 30, "%36") FB_T(14, 31, "0") FB_T(15, 31, "%36") FB_WAIT
                 : "=&v"(r[0]), "=&v"(r[1]), "=&v"(r[2]), "=&v"(r[3]), "=&v"(r[4]), "=&v"(r[5]), "=&v"(r[6]),
                   "=&v"(r[7]), "=&v"(r[8]), "=&v"(r[9]), "=&v"(r[10]), "=&v"(r[11]), "=&v"(r[12]), "=&v"(r[13]),
                   "=&v"(r[14]), "=&v"(r[15]), "=&v"(r[16]), "=&v"(r[17]), "=&v"(r[18]), "=&v"(r[19]), "=&v"(r[20]),
                   "=&v"(r[21]), "=&v"(r[22]), "=&v"(r[23])
                 : "v"(a[0]), "v"(a[1]), "v"(a[2]), "v"(a[3]), "v"(a[4]), "v"(a[5]), "v"(a[6]), "v"(a[7]), "v"(b[0]),
                   "v"(b[1]), "v"(b[2]), "v"(b[3]), "n"(SA), "n"(SB)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) A[i] = fb_join(r[2 * i], r[2 * i + 1]);
#pragma unroll
    for (int i = 0; i < 4; ++i) B[i] = fb_join(r[16 + 2 * i], r[17 + 2 * i]);
}

__device__ __forceinline__ uint32_t fb_lds(const uint8_t* p) {
    return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const uint8_t*)p;
}
// lane's byte in a KC stage for the 16 rows from 0 on
__device__ __forceinline__ uint32_t fb_frag_kc() {
    const int i = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
    return (uint32_t)(i * 64 + ((q ^ ((i >> 1) & 3)) * 16));
}
// lane's byte in an MC or MB stage of R columns for the 16 columns 16 t ..
template <FbLay LAY, int R>
__device__ __forceinline__ uint32_t fb_frag_mc(int t) {
    typedef FbCopy<LAY, R, R / 16> C;
    const int i = threadIdx.x & 15, q = (threadIdx.x & 63) >> 4;
    const int k = 8 * q + (i >> 2);
    if (LAY == FB_MB) return (uint32_t)((t >> 1) * 2048 + k * 64 + (((t & 1) ^ C::perm(k)) * 32) + 8 * (i & 3));
    return (uint32_t)(k * R * 2 + ((t ^ C::perm(k)) * 32) + 8 * (i & 3));
}

// acc += A B^T of a block of WM x WN waves, wave tiles of 16 MT rows by 16 NT columns.  PAIR: B's columns are two sides of
// half as many each, the second one's rows at b2 (a wave takes half of its columns from either).  The second operand
// goes into the MFMA first: lane (i, q) gets row 16 mi + i of its rows and four consecutive columns
// 4 q .. of block ni.  lds: kFbStages stages.  Every wave has passed its last read of lds before the call.
template <int WM, int WN, int MT, int NT>
struct FbShape {
    static constexpr int NW = WM * WN, BM = 16 * MT * WM, BN = 16 * NT * WN;
    static constexpr int STAGE = (BM + BN) * 64;
    static constexpr int LDS = kFbStages * STAGE;
};

template <int WM, int WN, int MT, int NT, FbLay AL, FbLay BL, bool PAIR = false>
__device__ __forceinline__ void fb_product(const FbSide& A, const FbSide& B, const uint16_t* b2, int64_t K, uint8_t* lds,
                                           floatx4 (&acc)[MT][NT]) {
    typedef FbShape<WM, WN, MT, NT> S;
    constexpr int RB = PAIR ? S::BN / 2 : S::BN;
    typedef FbCopy<AL, S::BM, S::NW> CA;
    typedef FbCopy<BL, RB, S::NW> CB;
    constexpr int LD = CA::N + CB::N * (PAIR ? 2 : 1);
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave / WN, wn = wave % WN;
    CA ca;
    CB cb;
    ca.start(A, wave);
    cb.start(B, wave);
    const FbSide B2{{b2, B.m.ld, B.m.gs, B.m.ts}, B.rows};
    const int steps = (int)((K + 31) / 32);
    auto issue = [&](int s, int slot) {
        uint8_t* d = lds + slot * S::STAGE;
        ca.issue(A, (int64_t)s * 32, K, d, wave);
        cb.issue(B, (int64_t)s * 32, K, d + CA::BYTES, wave);
        if (PAIR) cb.issue(B2, (int64_t)s * 32, K, d + CA::BYTES + CB::BYTES, wave);
    };
    uint32_t fa[AL == FB_KC ? 1 : MT], fb[BL == FB_KC ? 1 : 4];
    if constexpr (AL != FB_KC) {
#pragma unroll
        for (int t = 0; t < MT; ++t) fa[t] = fb_lds(lds) + fb_frag_mc<AL, S::BM>(MT * wm + t);
    } else {
        fa[0] = fb_lds(lds) + fb_frag_kc() + wm * MT * 1024;
    }
    if constexpr (BL == FB_KC) {
        fb[0] = fb_lds(lds) + CA::BYTES + fb_frag_kc() + wn * NT * 1024;
    } else if constexpr (!PAIR) {
#pragma unroll
        for (int t = 0; t < NT; ++t) fb[t] = fb_lds(lds) + CA::BYTES + fb_frag_mc<BL, RB>(NT * wn + t);
    } else {
#pragma unroll
        for (int t = 0; t < NT; ++t)
            fb[t] = fb_lds(lds) + CA::BYTES + (t < NT / 2 ? 0 : CB::BYTES) + fb_frag_mc<BL, RB>(NT / 2 * wn + t % (NT / 2));
    }
#pragma unroll
    for (int s = 0; s < kFbStages - 1; ++s)
        if (s < steps) issue(s, s);
    int slot = 0;
    for (int s = 0; s < steps; ++s) {
        if (s + kFbStages - 2 < steps) fb_wait<LD * (kFbStages - 2)>();
        else fb_wait<0>();
        fb_barrier();
        const int into = slot == 0 ? kFbStages - 1 : slot - 1;   // the stage of step s - 1
        if (s + kFbStages - 1 < steps) issue(s + kFbStages - 1, into);
        fbf16x8 a[MT], b[NT];
        const uint32_t at = (uint32_t)(slot * S::STAGE);
        if constexpr (BL == FB_KC) {
            fb_read_kk(fa[0] + at, fb[0] + at, a, b);
        } else {
            uint32_t vb[4];
#pragma unroll
            for (int t = 0; t < 4; ++t) vb[t] = fb[t] + at;
            if constexpr (AL != FB_KC) {
                uint32_t va[MT];
#pragma unroll
                for (int t = 0; t < MT; ++t) va[t] = fa[t] + at;
                fb_read_mm<CA::HALF, CB::HALF>(va, vb, a, b);
            } else {
                fb_read_km<CB::HALF>(fa[0] + at, vb, a, b);
            }
        }
#pragma unroll
        for (int mi = 0; mi < MT; ++mi)
#pragma unroll
            for (int ni = 0; ni < NT; ++ni)
                acc[mi][ni] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[ni], a[mi], acc[mi][ni], 0, 0, 0);
        slot = slot == kFbStages - 1 ? 0 : slot + 1;
    }
}

}  // namespace gsc
