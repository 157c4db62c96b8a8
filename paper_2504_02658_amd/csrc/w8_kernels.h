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
    int m_tiles, n_tiles;           // EPI 1, 2: m_tiles slots, some of them empty; the rest is set at the launch
    int group_m, span;              // order of the tiles (below)
    const int32_t* x_rows;          // EPI 1: token of a sorted row;  EPI 2: pair of a sorted row
    const float* gates;             // EPI 2: factor per pair
    void* out;                      // EPI 0: [M x N] 16-bit;  EPI 1: [rows x N] fp32;  EPI 2: [pairs x N] fp32
    int act_bf16;                   // EPI 0
};
// The kernels of a product, named by rows x features of a workgroup (EPI 1: half as many output features, from gate and up).
enum W8Kernel { W8_WIDE_16x16, W8_WIDE_16x32, W8_WIDE_16x64, W8_WIDE_32x32, W8_WIDE_32x64, W8_WIDE_64x64, W8_TILE_64x128, W8_TILE_128x128, W8_TILE_128x256 };
constexpr int64_t kW8MaxGroups = int64_t(1) << 22;      // workgroups of a product, of 512 threads at most: 2^31 work items
int launch_w8_product(const W8TileArgs& a, int epi, W8Kernel k, hipStream_t stream);
// Up to 16 rows whose codes fit kW8WideStaged bytes, in one launch: a.A is the 16-bit activations, k one of the kernels of 16 rows.  (Every
// workgroup quantizes all rows: N = 14336, K = 4096 takes 15.3 us in one launch against 17.6 in two for one row, 15.4 / 18.0 for four, 19.5 /
// 17.4 for eight; 16 rows of 1024 x 1024 5.9 / 8.0.)
constexpr int kW8WideStaged = 16 * 1024;
int launch_w8_staged(const W8TileArgs& a, W8Kernel k, hipStream_t stream);
int launch_w8_wide(const W8TileArgs& a, int epi, int tm, int rn, hipStream_t stream);      // w8_wide.hip: 16 tm x 16 rn


// Tile of a workgroup.  Workgroup i runs on XCD i % 8, each of which has an L2 of its own, so every XCD gets a contiguous range of
// an order in which tiles that share rows or columns are close: groups of group_m tiles of rows; inside a group runs of `span` columns;
// inside a run one tile of rows after the other.
__device__ __forceinline__ void w8_tile_of(uint32_t i, int m_tiles, int n_tiles, int group_m, int span, int* mt, int* nt) {
    const uint32_t total = (uint32_t)m_tiles * (uint32_t)n_tiles, x = i & 7u, per = total >> 3, rem = total & 7u;
    const uint32_t l = x * per + (x < rem ? x : rem) + (i >> 3);
    const uint32_t group = l / (uint32_t)(group_m * n_tiles), in = l - group * (uint32_t)(group_m * n_tiles);
    const uint32_t left = (uint32_t)m_tiles - group * (uint32_t)group_m, rows = left < (uint32_t)group_m ? left : (uint32_t)group_m;
    const uint32_t run = in / (rows * (uint32_t)span), at = in - run * rows * (uint32_t)span, n0 = run * (uint32_t)span;
    const uint32_t cols = (uint32_t)n_tiles - n0 < (uint32_t)span ? (uint32_t)n_tiles - n0 : (uint32_t)span, r = at / cols;
    *nt = (int)(n0 + at - r * cols);
    *mt = (int)(group * (uint32_t)group_m + r);
}


bool w8_shape_ok(int64_t N, int64_t K);

}  // namespace milo
