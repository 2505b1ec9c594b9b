// Feed-forward kernels for many rows of at most 256 channels on either side (bfloat16; ffn_res.hip), used by ffn.hip.
#pragma once

#include "row_vec.h"

namespace gsc {

constexpr int kResMax = 256;    // channels

// Bytes of the packed weights of either pass.
size_t res_pack_bytes(int ci, int f, int co);

// Y (n x co) = (act(X Wg) * (X Wu)) Wd, all rows at any address; pack: res_pack_bytes of device memory, 16-byte aligned.
void res_fwd(const uint16_t* X, int64_t n, int ci, const uint16_t* Wg, const uint16_t* Wu, int f, const uint16_t* Wd, int co,
             int act, uint16_t* Y, void* pack, hipStream_t s);

// H, dG and dU (row_blocks; columns behind f up to whole 64s zero); more than 64 channels on either side.
void res_mid(const uint16_t* X, const uint16_t* dY, int64_t n, int ci, const uint16_t* Wg, const uint16_t* Wu, int f,
             const uint16_t* Wd, int co, int act, RowMat<uint16_t> H, RowMat<uint16_t> dG, RowMat<uint16_t> dU, void* pack,
             hipStream_t s);

}  // namespace gsc
