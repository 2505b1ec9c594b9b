// Feed-forward kernels for many rows of at most 256 channels (bfloat16): a block keeps 128 rows of X as MFMA fragments
// in the registers of its eight waves and walks over the hidden columns, 64 at a time, while the weights stream through LDS
// stages that are filled two or three stages ahead.
//
// Against the tiles of ffn_bf16.h: a row is read once instead of once per 64 hidden columns, no tile starts with an empty
// pipeline, and k_ffn_fwd_res keeps the hidden rows in LDS: only X, Y and the weights (from the L2) move.
//
// The weights are first packed (k_ffn_pack) in the order in which the waves read them: blocks of 1 KiB that hold the 32
// columns x 16 reduction elements of a v_mfma_f32_32x32x16_bf16 operand, lane after lane (lane (c, h): column c,
// elements 8 h .. 8 h + 7), zeros behind the ends.  So copies into LDS are contiguous and need no masks, and a
// fragment is one 16-byte read per lane at a constant offset, which is started well before the product that needs it:
// every stage is an array of its own, so that the compiler can tell the copies into one from the reads of another.
//
// What bounds it: LDS reads, the matrix cores and the activation's vector instructions together (cycles below; the activation
// about 2,500), which overlap little.  The two waves of a SIMD pass the same barriers, so they would do the same at the same
// time; therefore the products of a chunk are interleaved with the activation of the chunk before it.
//
// Wave (m, n) of 4 x 2: rows 32 m .., hidden columns 32 n .. of a chunk; in the output projection output columns
// 16 TT n .. .  The MFMA takes the weights first: lane (i, h) of a 32 x 32 tile gets row i and columns 8 g + 4 h + e in
// register 4 g + e.
//
// 300,000 rows, 256 channels, 1,024 hidden: with the weights read as they lie by transpose reads in blocks of assembly that
// wait for themselves, 705 us forward and 835 us for k_ffn_mid_res; packed, without the interleaving, 597 and 840 us; as they
// are 568 and 722.  A chunk of 64 hidden columns costs a compute unit about 3,100 cycles of MFMA and, in 1 KiB fragments at
// 128 bytes a cycle, 3,300 (forward) and 4,096 cycles of LDS reads beside the activation, and takes about 8,500 and 10,800.
#include "ffn_res.h"

#include "ffn_act.h"
#include "ffn_mma.h"

namespace gsc {

constexpr int kResThreads = 512;
constexpr int kResRows = 128;

// Packed weights: for every chunk of 64 hidden columns the projections' blocks, by reduction step (KT of them, 16 elements each)
// the gate's and the other's columns 0 .. 31, then 32 .. 63 (4 KiB a step); after all chunks' of those, Wd's:
//   forward: by reduction step (4) its KT / 2 tiles of 32 output columns;  backward (Wd transposed): by reduction step
//   (KT) the two tiles of 32 hidden columns.  2 KiB per KT either way.
constexpr int res_pair_bytes(int KT) { return KT * 4096; }
constexpr int res_last_bytes(int KT) { return KT * 2048; }

struct ResPack {
    const uint16_t *g, *u, *d;   // c_in x f, c_in x f, f x c_out, as they are
    int ci, f, co, kt, back;
};

// One 16-byte piece a thread.
__global__ void __launch_bounds__(256) k_ffn_pack(ResPack p, uint16_t* __restrict__ out) {
    const int pair = res_pair_bytes(p.kt) / 16, last = res_last_bytes(p.kt) / 16;
    const int64_t chunks = (p.f + 63) / 64, pairs = chunks * pair;
    for (int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x; at < pairs + chunks * last; at += (int64_t)gridDim.x * 256) {
        const int64_t b = at < pairs ? at : at - pairs;
        const int ch = (int)(b / (at < pairs ? pair : last)), blk = (int)(b - (int64_t)ch * (at < pairs ? pair : last)) >> 6;
        const int c = (int)b & 31, h = (int)(b >> 5) & 1;
        const uint16_t* W = p.d;
        int k, col, kn, cn;          // reduction element, column, their ends
        int64_t sk, sc;              // ... and strides
        if (at < pairs) {
            W = blk & 1 ? p.u : p.g;
            k = (blk >> 2) * 16;
            col = ch * 64 + (blk >> 1 & 1) * 32 + c;
            kn = p.ci, cn = p.f, sk = p.f, sc = 1;
        } else if (p.back) {
            k = (blk >> 1) * 16;
            col = ch * 64 + (blk & 1) * 32 + c;
            kn = p.co, cn = p.f, sk = 1, sc = p.co;
        } else {
            const int tt = p.kt / 2;
            k = ch * 64 + blk / tt * 16;
            col = blk % tt * 32 + c;
            kn = p.f, cn = p.co, sk = p.co, sc = 1;
        }
        k += 8 * h;
        uint32_t v[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = k + e < kn && col < cn ? W[(k + e) * sk + col * sc] : 0u;
        reinterpret_cast<uint4*>(out)[at] = uint4{v[0] | v[1] << 16, v[2] | v[3] << 16, v[4] | v[5] << 16, v[6] | v[7] << 16};
    }
}

// Fragments of a wave's 32 rows: lane (i, h) holds row i, elements 16 k + 8 h .., below `cols`, from row-major memory at
// any address; steps k0, k0 + 1, ... .
template <int N>
__device__ __forceinline__ void res_rows(const uint16_t* __restrict__ X, int64_t ld, int cols, int64_t row0, int64_t n, int k0,
                                         fbf16x8 (&a)[N]) {
    const int i = threadIdx.x & 31, h = (threadIdx.x & 63) >> 5;
    const int64_t row = row0 + i;
    auto load = [&](auto TAIL) {
#pragma unroll
        for (int kk = 0; kk < N; ++kk) {
            const int k = 16 * (k0 + kk) + 8 * h;
            const RowVec<uint16_t>::Raw r =
                load_vec<uint16_t, decltype(TAIL)::value>(X + row * ld + k, row < n ? cols - k : 0);
            a[kk] = __builtin_bit_cast(fbf16x8, uint4{r[0], r[1], r[2], r[3]});
        }
    };
    if (cols % 8) load(std::true_type{});
    else load(std::false_type{});
}

// The stages: PS of a chunk's projections (32 KiB, or all of fewer steps) and one of its Wd, in a fixed order that repeats every
// U chunks = SLOTS stages, so that a stage's slot and the loads in flight behind it are known at compile time.  FIRST:
// projections that come before the order starts (forward: those of chunk 0, as chunk c + 1's come before chunk c's Wd).
template <int KT, int FIRST>
struct ResOrder {
    static constexpr int PS = KT > 8 ? KT / 8 : 1, PB = res_pair_bytes(KT) / PS, DB = res_last_bytes(KT);   // stages, bytes
    static constexpr int U = PS == 1 ? 2 : 1, SPC = PS + 1, SLOTS = U * SPC;
    static constexpr int KP = KT / PS;   // reduction steps of a projections' stage
    static constexpr bool last(int s) { return s >= FIRST && (s - FIRST) % SPC == PS; }
    static constexpr int loads(int s) { return (last(s) ? DB : PB) / 8192; }   // instructions of a wave
    // loads of the stages after s that have been started when s is read
    static constexpr int later(int s) {
        int n = 0;
        for (int k = 1; k < SLOTS - 1; ++k) n += loads(s + k);
        return n;
    }
};

// Copies into LDS of one wave.
template <typename O>
struct ResCopies {
    const uint8_t *pair, *last;   // next of either kind
    int pairs, lasts;             // left of either kind
    int wave;

    // Starts stage S (a number of the order).  Copies that carry nothing are started beyond the end, so that the number in
    // flight is the same everywhere: with branches around them the compiler cannot tell which have landed and waits for all
    // of them before it reads a stage.
    template <int S>
    __device__ __forceinline__ void start(uint8_t* dst) {
        constexpr int L = O::loads(S);
        int& left = O::last(S) ? lasts : pairs;
        const uint8_t*& src = O::last(S) ? last : pair;
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)src, (short)0, 0x7fffffff, kBufFlags);
        const uint32_t off = left > 0 ? (uint32_t)(wave * L * 1024 + (threadIdx.x & 63) * 16) : kBufNone;
#pragma unroll
        for (int j = 0; j < L; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(
                rs, (__attribute__((address_space(3))) void*)(dst + (wave * L + j) * 1024), 16, off + j * 1024, 0, 0, 0);
        --left;
        src += L * 8192;
    }
    // Until stage S has landed for all waves.  MORE: memory instructions of this wave since, other than copies (they retire in
    // order).  Every wave's LDS reads and writes before it are done, so what they read may be written again.
    template <int S, int MORE>
    __device__ __forceinline__ void wait() {
        fb_wait<O::later(S) + MORE>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        fb_barrier();
    }
};

#define RES_SLOTS(O)                                                                               \
    __shared__ __attribute__((aligned(1024))) uint8_t slot0[O::PB];                                \
    __shared__ __attribute__((aligned(1024))) uint8_t slot1[O::PB];                                \
    __shared__ __attribute__((aligned(1024))) uint8_t slot2[O::PB];                                \
    __shared__ __attribute__((aligned(1024))) uint8_t slot3[O::SLOTS > 3 ? O::PB : 16];            \
    auto slot = [&](auto N) -> uint8_t* {                                                          \
        constexpr int k = decltype(N)::value % O::SLOTS;                                           \
        return k == 0 ? slot0 : (k == 1 ? slot1 : (k == 2 ? slot2 : slot3));                       \
    };

struct ResPairFrag {
    fbf16x8 a, b;
};

// H, dG and dU of 128 rows and `per` hidden chunks from blockIdx.y * per on.  KT: 16-element steps of the
// wider of ci and co (8 or 16); W: the weights packed for it.  The block's dY lies in LDS as fragments (the registers
// hold X, a chunk's sums and those of the chunk before).
template <int KT, int ACT>
__global__ void __launch_bounds__(kResThreads, 1)
k_ffn_mid_res(const uint16_t* __restrict__ X, const uint16_t* __restrict__ dY, int64_t n, int ci, int co,
              const uint8_t* __restrict__ W, int f, RowMat<uint16_t> H, RowMat<uint16_t> dG, RowMat<uint16_t> dU, int per) {
    typedef ResOrder<KT, 0> O;
    RES_SLOTS(O)
    __shared__ __attribute__((aligned(1024))) uint8_t dys[4 * KT * 1024];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const int chunks_all = (f + 63) / 64, ch0 = blockIdx.y * per, chunks = min(per, chunks_all - ch0);
    const int64_t r0 = (int64_t)blockIdx.x * kResRows + 32 * wm;
    ResCopies<O> cp;
    cp.pair = W + (int64_t)ch0 * res_pair_bytes(KT);
    cp.last = W + (int64_t)chunks_all * res_pair_bytes(KT) + (int64_t)ch0 * res_last_bytes(KT);
    cp.pairs = chunks * O::PS;
    cp.lasts = chunks;
    cp.wave = wave;
    fbf16x8 x[KT];
    res_rows<KT>(X, ci, ci, r0, n, 0, x);
    uint8_t* dyw = dys + wm * KT * 1024;
    {
        fbf16x8 d[KT / 2];
        res_rows<KT / 2>(dY, co, co, r0, n, wn * (KT / 2), d);
#pragma unroll
        for (int k = 0; k < KT / 2; ++k)
            *reinterpret_cast<fbf16x8*>(dyw + (wn * (KT / 2) + k) * 1024 + (threadIdx.x & 63) * 16) = d[k];
    }
    res_each<O::SLOTS - 1>([&](auto N) { cp.template start<decltype(N)::value>(slot(N)); });
    floatx16 pg{}, pu{}, pd{};   // the chunk before: gates, partners and dH, then dG, dU and H
    uint32_t ph[8];
    auto epi = [&](int e) {
        float a, d;
        ffn_act<ACT, true, true>(pg[e], a, d);
        const float up = pu[e], g = pd[e];
        pd[e] = a * up;
        pg[e] = g * up * d;
        pu[e] = g * a;
    };
    // array k of the chunk before, as bfloat16 pairs
    auto put = [&](int k, int ch) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            ph[e] = k == 0 ? pack_bf16(pd[2 * e], pd[2 * e + 1])
                           : (k == 1 ? pack_bf16(pg[2 * e], pg[2 * e + 1]) : pack_bf16(pu[2 * e], pu[2 * e + 1]));
        // the wave's 32 rows of a block of 128 rows by 32 columns (rows behind the last one too: the blocks are whole)
        res_store<true>((k == 0 ? H : (k == 1 ? dG : dU)).at(r0, (int64_t)(ch0 + ch) * 64 + 32 * wn).p, 32, 0, 0, 0, 32, ph);
    };
    // Six stores follow the start of every chunk's last stage, so that the waits can count them: before the first chunk, and in
    // it, they write where its values come later.
#pragma unroll
    for (int k = 0; k < 3; ++k) put(k, 0);
    for (int cb = 0; cb < chunks; cb += O::U)
        res_each<O::U>([&](auto UU) {
            constexpr int u = decltype(UU)::value;
            const int ch = cb + u;
            if (ch >= chunks) return;
            floatx16 g{}, up{}, dh{};
            res_each<O::PS>([&](auto P) {
                constexpr int p = decltype(P)::value, S = u * O::SPC + p, E = 16 / O::PS / (2 * O::KP / 4);
                cp.template wait<S, 6>();
                cp.template start<S + O::SLOTS - 1>(slot(std::integral_constant<int, S + O::SLOTS - 1>{}));
                const uint8_t* b = slot(std::integral_constant<int, S>{}) + wn * 2048;
                res_stream<2 * O::KP, 4, 7>(
                    [&](int j) { return res_frag(b + (j >> 1) * 4096 + (j & 1) * 1024); },
                    [&](int j, fbf16x8 w) {
                        if (j & 1) up = res_mma(w, x[p * O::KP + (j >> 1)], up);
                        else g = res_mma(w, x[p * O::KP + (j >> 1)], g);
                    },
                    [&](auto I) {
#pragma unroll
                        for (int e = 0; e < E; ++e) epi(p * (16 / O::PS) + decltype(I)::value * E + e);
                    });
            });
            constexpr int S = u * O::SPC + O::PS;
            cp.template wait<S, O::PS == 1 ? 6 : 0>();
            cp.template start<S + O::SLOTS - 1>(slot(std::integral_constant<int, S + O::SLOTS - 1>{}));
            const uint8_t* b = slot(std::integral_constant<int, S>{}) + wn * 1024;
#pragma unroll
            for (int k = 0; k < 3; ++k) put(k, ch > 0 ? ch - 1 : 0);
            res_stream<KT, 4, 0>([&](int j) { return ResPairFrag{res_frag(b + j * 2048), res_frag(dyw + j * 1024)}; },
                                 [&](int j, const ResPairFrag& w) { dh = res_mma(w.a, w.b, dh); }, [](auto) {});
            pg = g;
            pu = up;
            pd = dh;
        });
    fb_wait<0>();   // no copy is in flight when the block ends
#pragma unroll
    for (int e = 0; e < 16; ++e) epi(e);
#pragma unroll
    for (int k = 0; k < 3; ++k) put(k, chunks - 1);
}

// Y (n x co) of 128 rows.  KT: 16-element steps of the wider of ci and co (4, 8 or 16).  The hidden rows of a chunk pass
// through LDS (rows of 128 bytes, piece c of row r at c ^ (r & 7)) while the next chunk's are worked out.
template <int KT, int ACT>
__global__ void __launch_bounds__(kResThreads, 1)
k_ffn_fwd_res(const uint16_t* __restrict__ X, int64_t n, int ci, int co, const uint8_t* __restrict__ W, int f,
              uint16_t* __restrict__ Y) {
    constexpr int TT = KT / 2, TW = TT / 2;   // tiles of 32 output columns, of a wave
    typedef ResOrder<KT, (KT > 8 ? KT / 8 : 1)> O;
    RES_SLOTS(O)
    __shared__ __attribute__((aligned(1024))) uint8_t hid[kResRows * 128];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wm = wave >> 1, wn = wave & 1;
    const int row = 32 * wm + (threadIdx.x & 31), h = (threadIdx.x & 63) >> 5;
    const int chunks = (f + 63) / 64;
    const int64_t r0 = (int64_t)blockIdx.x * kResRows + 32 * wm;
    ResCopies<O> cp;
    cp.pair = W;
    cp.last = W + (int64_t)chunks * res_pair_bytes(KT);
    cp.pairs = chunks * O::PS;
    cp.lasts = chunks;
    cp.wave = wave;
    fbf16x8 x[KT];
    res_rows<KT>(X, ci, ci, r0, n, 0, x);
    floatx16 y[TW];
#pragma unroll
    for (int t = 0; t < TW; ++t) y[t] = floatx16{};
    res_each<O::SLOTS - 1>([&](auto N) { cp.template start<decltype(N)::value>(slot(N)); });
    floatx16 g{}, up{}, pg, pu;
    float v[4];
    auto epi = [&](int e) {
        float a, d;
        ffn_act<ACT, false, true>(pg[e], a, d);
        v[e & 3] = a * pu[e];
        if ((e & 3) == 3)   // columns 32 wn + 8 j + 4 h .., j = e / 4: half of piece 4 wn + j
            *reinterpret_cast<uint2*>(hid + row * 128 + (((4 * wn + (e >> 2)) ^ (row & 7)) * 16) + h * 8) =
                uint2{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3])};
    };
    // stage S: projections p of a chunk, with a share of the activation of the chunk before
    auto pairs = [&](auto SS, auto P, bool more, auto side) {
        constexpr int S = decltype(SS)::value, p = decltype(P)::value;
        cp.template wait<S, 0>();
        cp.template start<S + O::SLOTS - 1>(slot(std::integral_constant<int, S + O::SLOTS - 1>{}));
        const uint8_t* b = slot(std::integral_constant<int, S>{}) + wn * 2048;
        if (more)
            res_stream<2 * O::KP, 4, 6>(
                [&](int j) { return res_frag(b + (j >> 1) * 4096 + (j & 1) * 1024); },
                [&](int j, fbf16x8 w) {
                    if (j & 1) up = res_mma(w, x[p * O::KP + (j >> 1)], up);
                    else g = res_mma(w, x[p * O::KP + (j >> 1)], g);
                },
                side);
        else
            res_each<2 * O::KP / 4>(side);
    };
    res_each<O::PS>([&](auto P) { pairs(P, P, true, [](auto) {}); });
    for (int cb = 0; cb < chunks; cb += O::U)
        res_each<O::U>([&](auto UU) {
            constexpr int u = decltype(UU)::value, S0 = O::PS + u * O::SPC;
            const int ch = cb + u;
            if (ch >= chunks) return;
            const bool more = ch + 1 < chunks;
            pg = g;
            pu = up;
            g = floatx16{};
            up = floatx16{};
            res_each<O::PS>([&](auto P) {
                constexpr int p = decltype(P)::value, E = 16 / O::PS / (2 * O::KP / 4);
                pairs(std::integral_constant<int, S0 + p>{}, P, more, [&](auto I) {
#pragma unroll
                    for (int e = 0; e < E; ++e) epi(p * (16 / O::PS) + decltype(I)::value * E + e);
                });
            });
            constexpr int S = S0 + O::PS;
            cp.template wait<S, 0>();
            cp.template start<S + O::SLOTS - 1>(slot(std::integral_constant<int, S + O::SLOTS - 1>{}));
            const uint8_t* b = slot(std::integral_constant<int, S>{}) + wn * TW * 1024;
            fbf16x8 a[4];
#pragma unroll
            for (int k = 0; k < 4; ++k)
                a[k] = *reinterpret_cast<const fbf16x8*>(hid + row * 128 + (((2 * k + h) ^ (row & 7)) * 16));
            res_stream<4 * TW, 4, 0>([&](int j) { return res_frag(b + (j / TW * TT + j % TW) * 1024); },
                                     [&](int j, fbf16x8 w) { y[j % TW] = res_mma(w, a[j / TW], y[j % TW]); }, [](auto) {});
        });
    fb_wait<0>();   // no copy is in flight when the block ends
#pragma unroll
    for (int t = 0; t < TW; ++t) {
        uint32_t o[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) o[e] = pack_bf16(y[t][2 * e], y[t][2 * e + 1]);
        res_store<false>(Y, co, r0, n, 16 * TT * wn + 32 * t, co, o);
    }
}

static int res_steps(int ci, int co) {
    const int c = ci > co ? ci : co;
    return c <= 64 ? 4 : (c <= 128 ? 8 : 16);
}

size_t res_pack_bytes(int ci, int f, int co) {
    const int kt = res_steps(ci, co);
    return (size_t)((f + 63) / 64) * (res_pair_bytes(kt) + res_last_bytes(kt));
}

static int res_pack(int ci, int f, int co, const uint16_t* Wg, const uint16_t* Wu, const uint16_t* Wd, int back, void* pack,
                    hipStream_t s) {
    const int kt = res_steps(ci, co);
    const ResPack p{Wg, Wu, Wd, ci, f, co, kt, back};
    const size_t blocks = (res_pack_bytes(ci, f, co) + 4095) / 4096;
    hipLaunchKernelGGL(k_ffn_pack, dim3((unsigned)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, s, p,
                       reinterpret_cast<uint16_t*>(pack));
    return kt;
}

// f(KT (at least LEAST), activation as constants)
template <int LEAST, typename F>
static void res_with(int kt, int act, F f) {
    auto with = [&](auto KT) {
        switch (act) {
            case GSC_GATE_RELU: return f(KT, std::integral_constant<int, GSC_GATE_RELU>{});
            case GSC_GATE_SIGMOID: return f(KT, std::integral_constant<int, GSC_GATE_SIGMOID>{});
            case GSC_GATE_GELU: return f(KT, std::integral_constant<int, GSC_GATE_GELU>{});
            case GSC_GATE_GELU_TANH: return f(KT, std::integral_constant<int, GSC_GATE_GELU_TANH>{});
            default: return f(KT, std::integral_constant<int, GSC_GATE_SILU>{});
        }
    };
    if constexpr (LEAST <= 4)
        if (kt == 4) return with(std::integral_constant<int, 4>{});
    if (kt == 8) with(std::integral_constant<int, 8>{});
    else with(std::integral_constant<int, 16>{});
}

void res_fwd(const uint16_t* X, int64_t n, int ci, const uint16_t* Wg, const uint16_t* Wu, int f, const uint16_t* Wd, int co,
             int act, uint16_t* Y, void* pack, hipStream_t s) {
    res_with<4>(res_pack(ci, f, co, Wg, Wu, Wd, 0, pack, s), act, [&](auto KT, auto ACT) {
        auto* kern = k_ffn_fwd_res<decltype(KT)::value, decltype(ACT)::value>;
        hipLaunchKernelGGL(kern, dim3((unsigned)((n + kResRows - 1) / kResRows)), dim3(kResThreads), 0, s, X, n, ci, co,
                           reinterpret_cast<const uint8_t*>(pack), f, Y);
    });
}

// Hidden chunks are split over blocks where the row tiles are fewer than two a compute unit.
void res_mid(const uint16_t* X, const uint16_t* dY, int64_t n, int ci, const uint16_t* Wg, const uint16_t* Wu, int f,
             const uint16_t* Wd, int co, int act, RowMat<uint16_t> H, RowMat<uint16_t> dG, RowMat<uint16_t> dU, void* pack,
             hipStream_t s) {
    const int64_t tiles = (n + kResRows - 1) / kResRows, chunks = (f + 63) / 64;
    const int64_t parts = tiles >= 512 ? 1 : (512 + tiles - 1) / tiles;
    const int per = (int)((chunks + parts - 1) / parts);
    res_with<8>(res_pack(ci, f, co, Wg, Wu, Wd, 1, pack, s), act, [&](auto KT, auto ACT) {
        auto* kern = k_ffn_mid_res<decltype(KT)::value, decltype(ACT)::value>;
        hipLaunchKernelGGL(kern, dim3((unsigned)tiles, (unsigned)((chunks + per - 1) / per)), dim3(kResThreads), 0, s, X, dY, n,
                           ci, co, reinterpret_cast<const uint8_t*>(pack), f, H, dG, dU, per);
    });
}

}  // namespace gsc
