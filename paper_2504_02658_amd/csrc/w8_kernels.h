// Argument blocks and host-side launchers of the 8-bit integer path (internal to the library).
#pragma once

#include "milo_kernels.h"
#include "w8_device.h"

namespace milo {

// One packed weight (milo_pack_w8): blocked codes, then one fp32 scale per padded row.
__host__ __device__ inline const float* w8_scales(const void* w8, int64_t N, int64_t K) {
    return reinterpret_cast<const float*>(reinterpret_cast<const char*>(w8) + w8_code_bytes(N, K));
}

// Quantizes `rows` rows of K elements; `blocked`: into the blocked layout (and zeros up to whole blocks of rows), else
// row-major with `kblocks * 64` bytes per row.
struct W8QuantArgs {
    const void* in;
    int64_t rows, K;
    uint8_t* codes;
    float* scales;
    int blocked;
};
int launch_w8_quant(const W8QuantArgs& a, int in, hipStream_t stream);

// Tiled product.  Row r of a tile's A operand:
//   EPI 0 (a linear):         blocked activations, row 'tile * BM + r' of M
//   EPI 1 (gate and up):      row-major activations, row x_rows[row0 + r]
//   EPI 2 (down projection):  row-major codes of the SwiGLU output, row row0 + r
struct W8TileArgs {
    const uint8_t* A;
    uint64_t a_bytes;
    const float* a_scales;
    int64_t M, N, K;
    const void* w;                  // EPI 0
    const milo_w8_expert* experts;  // EPI 1, 2: device table
    const TileDesc* tiles;
    int m_tiles, n_tiles;           // EPI 1, 2: m_tiles slots, some of them empty; the rest is set by launch_w8_tile
    const int32_t* x_rows;          // EPI 1: token of a sorted row;  EPI 2: pair of a sorted row
    const float* gates;             // EPI 2: factor per pair
    void* out;                      // EPI 0: [M x N] 16-bit;  EPI 1: [rows x N] fp32;  EPI 2: [pairs x N] fp32
    int act_bf16;
};
int launch_w8_tile(const W8TileArgs& a, int epi, int bm, hipStream_t stream);

bool w8_shape_ok(int64_t N, int64_t K);

}  // namespace milo
