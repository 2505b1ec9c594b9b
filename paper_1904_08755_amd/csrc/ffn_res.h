// Feed-forward kernels that keep rows in registers, for many rows of few channels, used by ffn.hip: bfloat16 (ffn_res.hip) and
// float32 (ffn_res_f32.hip).
#pragma once

#include "row_vec.h"

namespace gsc {

constexpr int kResMax = 256, kResMaxF32 = 128;    // channels on either side

// Bytes of the packed weights of either pass.
size_t res_pack_bytes(int ci, int f, int co);

// Y (n x co) = (act(X Wg) * (X Wu)) Wd, all rows at any address; pack: res_pack_bytes of device memory, 16-byte aligned.
void res_fwd(const uint16_t* X, int64_t n, int ci, const uint16_t* Wg, const uint16_t* Wu, int f, const uint16_t* Wd, int co,
             int act, uint16_t* Y, void* pack, hipStream_t s);

// H, dG and dU (row_blocks; columns behind f up to whole 64s zero); more than 64 channels on either side.
void res_mid(const uint16_t* X, const uint16_t* dY, int64_t n, int ci, const uint16_t* Wg, const uint16_t* Wu, int f,
             const uint16_t* Wd, int co, int act, RowMat<uint16_t> H, RowMat<uint16_t> dG, RowMat<uint16_t> dU, void* pack,
             hipStream_t s);

// float32: Y; H, dG and dU as above (fp: f in whole 64s) and, unless null, dX.
void res_fwd(const float* X, int64_t n, int ci, const float* Wg, const float* Wu, int f, const float* Wd, int co, int act,
             float* Y, hipStream_t s);
void res_bwd(const float* X, const float* dY, int64_t n, int ci, const float* Wg, const float* Wu, int f, const float* Wd,
             int co, int act, int fp, RowMat<float> H, RowMat<float> dG, RowMat<float> dU, float* dX, hipStream_t s);

}  // namespace gsc
