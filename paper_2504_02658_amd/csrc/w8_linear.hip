// Linears in 8-bit integers: milo_pack_w8, milo_w8a8_gemm and the tiled product that the MoE layer shares.
#include <type_traits>

#include "milo_host.h"
#include "w8_kernels.h"

namespace milo {

// A row's sums have to fit 32 bits: 127 * 127 * K < 2^31.
constexpr int64_t kW8MaxK = 1 << 17;

bool w8_shape_ok(int64_t N, int64_t K) {
    return N >= 1 && K >= 1 && K <= kW8MaxK && N <= (int64_t(1) << 23) && N <= (int64_t(1) << 40) / K;
}

// ---------------------------------------------------------------------------------------------
// Row quantizer: a row is read once for its largest magnitude and, while it fits the registers of its TPR threads,
// quantized from there.
constexpr int kQuantThreads = 256, kQuantHeld = 4;
template <int IN, int TPR, bool BLOCKED>
__global__ __launch_bounds__(kQuantThreads) void w8_quant_kernel(const W8QuantArgs a, int kb) {
    constexpr int SZ = IN == W8_F32 ? 4 : 2;
    __shared__ uint32_t s_top[kQuantThreads / 64];
    const int tid = threadIdx.x % TPR;
    const int64_t row = (int64_t)blockIdx.x * (kQuantThreads / TPR) + threadIdx.x / TPR;
    const bool there = row < a.rows;
    const char* in = reinterpret_cast<const char*>(a.in) + (there ? row : 0) * a.K * SZ;
    const int64_t K = there ? a.K : 0;          // (rows beyond the last are all zero)
    const int pieces = kb * 4;                  // of 16 columns, with the padding
    W8Raw<IN> held[kQuantHeld];
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < kQuantHeld; ++i) {
        const int p = tid + i * TPR;
        held[i] = load16<IN>(in, (int64_t)p * 16, p < pieces ? K : 0);
    }
#pragma unroll
    for (int i = 0; i < kQuantHeld; ++i) top = raw_top<IN>(held[i], top);
    for (int p = tid + kQuantHeld * TPR; p < pieces; p += TPR) top = raw_top<IN>(load16<IN>(in, (int64_t)p * 16, K), top);
    top = wave_max(top);
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kQuantThreads / 64; ++w) top = s_top[w] > top ? s_top[w] : top;
    }
    const RowStep st = row_step(top);
    if (!there && !BLOCKED) return;
    auto put = [&](int p, const W8Raw<IN>& r) {
        float v[16];
        raw_values<IN>(r, v);
        const u32x4 c = row_codes16(v, st);
        uint8_t* to = BLOCKED ? a.codes + ((row >> 4) * kb + (p >> 2)) * 1024 + (p & 3) * 256 + (row & 15) * 16
                              : a.codes + row * kb * 64 + (int64_t)p * 16;
        *reinterpret_cast<u32x4*>(to) = c;
    };
#pragma unroll
    for (int i = 0; i < kQuantHeld; ++i)
        if (tid + i * TPR < pieces) put(tid + i * TPR, held[i]);
    for (int p = tid + kQuantHeld * TPR; p < pieces; p += TPR) put(p, load16<IN>(in, (int64_t)p * 16, K));
    if (tid == 0) a.scales[row] = st.s;
}

template <int IN, bool BLOCKED>
static int launch_quant(const W8QuantArgs& a, hipStream_t stream) {
    const int kb = (int)w8_kblocks(a.K);
    const int64_t rows = BLOCKED ? w8_rblocks(a.rows) * 16 : a.rows;
    if (rows == 0) return MILO_OK;
    if (kb * 4 <= 64 * kQuantHeld)      // a wave holds the whole row
        w8_quant_kernel<IN, 64, BLOCKED><<<dim3((unsigned)((rows + 3) / 4)), dim3(kQuantThreads), 0, stream>>>(a, kb);
    else
        w8_quant_kernel<IN, 256, BLOCKED><<<dim3((unsigned)rows), dim3(kQuantThreads), 0, stream>>>(a, kb);
    return launch_status();
}
int launch_w8_quant(const W8QuantArgs& a, int in, hipStream_t stream) {
    switch (in * 2 + (a.blocked ? 1 : 0)) {
        case 2 * W8_F32: return launch_quant<W8_F32, false>(a, stream);
        case 2 * W8_F32 + 1: return launch_quant<W8_F32, true>(a, stream);
        case 2 * W8_F16: return launch_quant<W8_F16, false>(a, stream);
        case 2 * W8_F16 + 1: return launch_quant<W8_F16, true>(a, stream);
        case 2 * W8_BF16: return launch_quant<W8_BF16, false>(a, stream);
        default: return launch_quant<W8_BF16, true>(a, stream);
    }
}

// ---------------------------------------------------------------------------------------------
// Up to 16 rows: the weight's bytes bound the call.  A workgroup owns 16 output features, its waves share K chunk by
// chunk (integer sums, so the split changes nothing), and each fragment of the weight goes from memory to the matrix
// core's operand registers as it is.
constexpr int kStreamWaves = 8;
template <bool BF>
__global__ __launch_bounds__(kStreamWaves * 64) void w8_stream_kernel(const uint8_t* __restrict__ xq, const float* __restrict__ xs, int64_t M, int64_t N, int64_t K,
                                                                      const uint8_t* __restrict__ w, uint16_t* __restrict__ out) {
    __shared__ i32x4 s_part[kStreamWaves][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kb = (int)w8_kblocks(K);
    const u32x4* const wp = reinterpret_cast<const u32x4*>(w + (int64_t)blockIdx.x * kb * 1024) + lane;
    const u32x4* const xp = reinterpret_cast<const u32x4*>(xq) + lane;
    i32x4 acc = {0, 0, 0, 0};
#pragma unroll 8
    for (int b = wave; b < kb; b += kStreamWaves) acc = mfma16_i8(wp[(int64_t)b * 64], xp[(int64_t)b * 64], acc);
    s_part[wave][lane] = acc;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 1; i < kStreamWaves; ++i) acc += s_part[i][lane];
    const int m = lane & 15;
    const int64_t n = (int64_t)blockIdx.x * 16 + (lane >> 4) * 4;
    if (m >= M || n >= N) return;
    const float* sw = w8_scales(w, N, K) + n;
    const float sx = xs[m];
    float v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = (float)acc[i] * sx * sw[i];
    store4<BF>(out + m * N + n, v, (int)(N - n < 4 ? N - n : 4), (N & 3) == 0);
}

// ---------------------------------------------------------------------------------------------
// Tile of a workgroup.  Workgroup i runs on XCD i % 8, each of which has an L2 of its own, so every XCD gets a contiguous range of
// an order in which tiles that share rows or columns are close: groups of kGroupM tiles of rows, and inside a group all columns,
// rows fastest.
constexpr int kGroupM = 8;
__device__ __forceinline__ void tile_of(uint32_t i, int m_tiles, int n_tiles, int* mt, int* nt) {
    const uint32_t total = (uint32_t)m_tiles * (uint32_t)n_tiles, x = i & 7u, per = total >> 3, rem = total & 7u;
    const uint32_t l = x * per + (x < rem ? x : rem) + (i >> 3);
    const uint32_t group = l / (uint32_t)(kGroupM * n_tiles), in = l - group * (uint32_t)(kGroupM * n_tiles);
    const uint32_t left = (uint32_t)m_tiles - group * kGroupM, rows = left < kGroupM ? left : kGroupM;
    *nt = (int)(in / rows);
    *mt = (int)(group * kGroupM + in % rows);
}

// The tiled product.
template <int WM, int WN, int TM, int TN, int NS, int EPI, bool BF>
__global__ __launch_bounds__(WM * WN * 64) void w8_tile_kernel(const W8TileArgs a) {
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32, NW = WM * WN;
    constexpr int ABLK = BM / 16, BBLK = BN / 16;       // 1-KB blocks of a stage (64 columns)
    constexpr int PA = ABLK / NW, PB = BBLK / NW;       // of them, copied by one wave
    constexpr int STAGE = (ABLK + BBLK) * 1024;
    constexpr int OUTN = EPI == 1 ? BN / 2 : BN;        // output columns of a tile
    static_assert(ABLK % NW == 0 && (EPI == 1 ? BBLK / 2 : BBLK) % NW == 0, "every wave copies as many blocks");
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int kb = (int)w8_kblocks(a.K);
    int mt, nt;
    tile_of(blockIdx.x, a.m_tiles, a.n_tiles, &mt, &nt);
    const int64_t n0 = (int64_t)nt * OUTN;
    int64_t row0;
    int rows;
    const uint8_t* w0;
    const uint8_t* w1;
    if constexpr (EPI == 0) {
        row0 = (int64_t)mt * BM;
        rows = (int)(a.M - row0 < BM ? a.M - row0 : BM);
        w0 = w1 = reinterpret_cast<const uint8_t*>(a.w);
    } else {
        const TileDesc t = a.tiles[mt];
        row0 = t.row0;
        rows = t.rows;
        if (rows == 0) return;
        const milo_w8_expert& e = a.experts[t.expert];
        w0 = reinterpret_cast<const uint8_t*>(EPI == 1 ? e.w1 : e.w2);
        w1 = reinterpret_cast<const uint8_t*>(EPI == 1 ? e.w3 : e.w2);
    }
    // where this wave's copies come from: activations, then the weight (gate and up: half of the rows each)
    const uint64_t wbytes = (uint64_t)w8_code_bytes(a.N, a.K), wskip = (uint64_t)(n0 >> 4) * kb * 1024;
    const uint64_t abase = EPI == 0 ? (uint64_t)row0 / 16 * kb * 1024 : 0;
    const BufRsrc ra = make_rsrc(a.A + abase, a.a_bytes - abase);
    const BufRsrc rb0 = make_rsrc(w0 + wskip, wbytes - wskip), rb1 = make_rsrc(w1 + wskip, wbytes - wskip);
    uint32_t aoff[PA], boff[PB];
#pragma unroll
    for (int i = 0; i < PA; ++i) {
        const int b = wave + i * NW;
        if constexpr (EPI == 0) {
            aoff[i] = (uint32_t)(b * kb) * 1024u + lane * 16;
        } else {
            int r = b * 16 + (lane & 15);
            r = (int)row0 + (r < rows ? r : 0);         // (rows beyond the tile's: computed, not stored)
            const int64_t src = EPI == 1 ? a.x_rows[r] : r;
            aoff[i] = (uint32_t)(src * kb * 64) + (lane >> 4) * 16;
        }
    }
#pragma unroll
    for (int i = 0; i < PB; ++i) boff[i] = (uint32_t)(((wave + i * NW) % (OUTN / 16)) * kb) * 1024u + lane * 16;
    auto issue = [&](int c) {
        unsigned char* const to = smem + (c % NS) * STAGE + wave * 1024;
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const uint32_t o = aoff[i];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LdsDst)(to + i * NW * 1024), 16, o, 0, 0, 0);
            aoff[i] += EPI == 0 ? 1024u : 64u;
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const uint32_t o = boff[i];
            if (EPI == 1 && i >= PB / 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rb1, (LdsDst)(to + (ABLK + i * NW) * 1024), 16, o, 0, 0, 0);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(rb0, (LdsDst)(to + (ABLK + i * NW) * 1024), 16, o, 0, 0, 0);
            boff[i] += 1024u;
        }
    };
    const int wm = wave % WM, wn = wave / WM, l32 = lane & 31, h = lane >> 5;
    const int frag = (l32 >> 4) * 1024 + h * 256 + (l32 & 15) * 16;
    i32x16 acc[TN][TM];
#pragma unroll
    for (int n = 0; n < TN; ++n)
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[n][m][i] = 0;
    // rows (of 32) of the weight's part of a stage that the wave's n-th tile reads
    auto brow = [&](int n) { return EPI == 1 ? (n < TN / 2 ? wn * (TN / 2) + n : OUTN / 32 + wn * (TN / 2) + n - TN / 2) : wn * TN + n; };
    // A stage is 64 columns, two steps of 32.  While the matrix cores work on one step the fragments of the next one are on their
    // way from LDS.  The copies of a wave complete in order: with at most those of the NS - 2 younger stages outstanding, stage
    // c + 1 is there; the barrier says so for all waves, and that all have read what they need of stage c, whose place the next
    // copies take.
    u32x4 af[2][TM], bf[2][TN];
    auto read = [&](int c, int k) {
        const unsigned char* const as = smem + (c % NS) * STAGE + wm * TM * 2048 + frag + k * 512;
        const unsigned char* const bs = smem + (c % NS) * STAGE + ABLK * 1024 + frag + k * 512;
#pragma unroll
        for (int n = 0; n < TN; ++n) bf[k][n] = *reinterpret_cast<const u32x4*>(bs + brow(n) * 2048);
#pragma unroll
        for (int m = 0; m < TM; ++m) af[k][m] = *reinterpret_cast<const u32x4*>(as + m * 2048);
    };
    auto multiply = [&](int k) {
#pragma unroll
        for (int m = 0; m < TM; ++m)
#pragma unroll
            for (int n = 0; n < TN; ++n) acc[n][m] = mfma32_i8(bf[k][n], af[k][m], acc[n][m]);
    };
    // one LDS read behind each of the first matrix instructions, instead of all of them in front
    auto mix = [&] {
#pragma unroll
        for (int i = 0; i < TM + TN; ++i) {
            __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
            __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(0x8, TM * TN - TM - TN, 0);
        __builtin_amdgcn_sched_barrier(0);
    };
    auto arrive = [&](auto counted, bool all) {
        if (!decltype(counted)::value && all) wait_vmem();
        else MILO_WAIT_VMEM((NS - 2) * (PA + PB));
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    };
    for (int c = 0; c < NS - 1 && c < kb; ++c) issue(c);
    arrive(std::bool_constant<false>{}, kb < NS - 1);
    if (NS - 1 < kb) issue(NS - 1);
    read(0, 0);
    int c = 0;
    auto stage = [&](auto more) {           // more: stage c + NS exists
        read(c, 1);
        multiply(0);
        mix();
        arrive(more, true);
        if constexpr (decltype(more)::value) issue(c + NS);
        read(c + 1, 0);                     // (behind the last stage: of no use)
        multiply(1);
        mix();
    };
    for (; c + NS < kb; ++c) stage(std::bool_constant<true>{});
    for (; c < kb; ++c) stage(std::bool_constant<false>{});
    // lane: row (of 32) l32, output features 8 i + 4 h + 0..3
    const bool vec = (a.N & 3) == 0;
    const auto sw0 = global_float(w8_scales(w0, a.N, a.K)), sw1 = global_float(w8_scales(w1, a.N, a.K));
#pragma unroll
    for (int m = 0; m < TM; ++m) {
        const int r = (wm * TM + m) * 32 + l32;
        if (r >= rows) continue;
        const int64_t row = row0 + r;
        float sx;
        int64_t to = row;
        if constexpr (EPI == 0) sx = a.a_scales[row];
        else if constexpr (EPI == 1) sx = a.a_scales[a.x_rows[row]];
        else {
            to = a.x_rows[row];
            sx = a.a_scales[row] * a.gates[to];
        }
#pragma unroll
        for (int n = 0; n < (EPI == 1 ? TN / 2 : TN); ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int64_t col = n0 + (EPI == 1 ? wn * (TN / 2) + n : wn * TN + n) * 32 + 8 * i + 4 * h;
                if (col >= a.N) continue;
                const int left = (int)(a.N - col < 4 ? a.N - col : 4);
                float v[4];
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    v[j] = (float)acc[n][m][4 * i + j] * sx * sw0[col + j];
                    if constexpr (EPI == 1) v[j] = silu_times(v[j], (float)acc[n + TN / 2][m][4 * i + j] * sx * sw1[col + j]);
                }
                if constexpr (EPI == 0) {
                    store4<BF>(reinterpret_cast<uint16_t*>(a.out) + to * a.N + col, v, left, vec);
                } else {
                    float* o = reinterpret_cast<float*>(a.out) + to * a.N + col;
                    if (vec) *reinterpret_cast<f32x4*>(o) = f32x4{v[0], v[1], v[2], v[3]};
                    else
                        for (int j = 0; j < left; ++j) o[j] = v[j];
                }
            }
    }
}

template <int WM, int WN, int TM, int TN, int NS, int EPI, bool BF>
static int launch_tile(W8TileArgs a, hipStream_t stream) {
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32, OUTN = EPI == 1 ? BN / 2 : BN, lds = NS * (BM + BN) * 64;
    if constexpr (lds > 64 * 1024) {
        static bool raised[64] = {false};
        int dev = 0;
        if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev >= 64) return MILO_ERR_HIP;
        if (!raised[dev]) {
            if (hipFuncSetAttribute(reinterpret_cast<const void*>(w8_tile_kernel<WM, WN, TM, TN, NS, EPI, BF>), hipFuncAttributeMaxDynamicSharedMemorySize, lds) != hipSuccess)
                return MILO_ERR_HIP;
            raised[dev] = true;
        }
    }
    if (EPI == 0) a.m_tiles = (int)((a.M + BM - 1) / BM);
    a.n_tiles = (int)((a.N + OUTN - 1) / OUTN);
    if ((int64_t)a.m_tiles * a.n_tiles > (int64_t(1) << 31) / (WM * WN * 64)) return MILO_ERR_SHAPE;
    w8_tile_kernel<WM, WN, TM, TN, NS, EPI, BF><<<dim3((unsigned)(a.m_tiles * a.n_tiles)), dim3(WM * WN * 64), lds, stream>>>(a);
    return launch_status();
}
template <int EPI, bool BF>
static int launch_tile_bm(const W8TileArgs& a, int bm, hipStream_t stream) {
    if (bm == 256) return launch_tile<2, 4, 4, 2, 4, EPI, BF>(a, stream);
    return launch_tile<2, 2, 2, 2, 4, EPI, BF>(a, stream);
}
int launch_w8_tile(const W8TileArgs& a, int epi, int bm, hipStream_t stream) {
    if (epi == 0) return a.act_bf16 ? launch_tile_bm<0, true>(a, bm, stream) : launch_tile_bm<0, false>(a, bm, stream);
    return epi == 1 ? launch_tile_bm<1, false>(a, bm, stream) : launch_tile_bm<2, false>(a, bm, stream);
}

}  // namespace milo

using namespace milo;

extern "C" size_t milo_w8_packed_bytes(int64_t N, int64_t K) {
    if (!w8_shape_ok(N, K)) return 0;
    return (size_t)w8_code_bytes(N, K) + (size_t)w8_rblocks(N) * 16 * sizeof(float);
}

extern "C" int milo_pack_w8(const void* W, int dtype, int64_t N, int64_t K, void* w8, void* stream) {
    if (!W || !w8) return MILO_ERR_NULL;
    if (!w8_shape_ok(N, K) || dtype < MILO_F32 || dtype > MILO_BF16) return MILO_ERR_SHAPE;
    if (!aligned16(W) || !aligned16(w8)) return MILO_ERR_ALIGN;
    W8QuantArgs a;
    a.in = W;
    a.rows = N;
    a.K = K;
    a.codes = reinterpret_cast<uint8_t*>(w8);
    a.scales = const_cast<float*>(w8_scales(w8, N, K));
    a.blocked = 1;
    return launch_w8_quant(a, dtype, (hipStream_t)stream);
}

static size_t gemm_scales_off(int64_t M, int64_t K) { return align_up((size_t)w8_code_bytes(M, K), 256); }

extern "C" size_t milo_w8a8_gemm_workspace(int64_t M, int64_t N, int64_t K) {
    if (M < 1 || !w8_shape_ok(N, K) || !w8_shape_ok(M, K)) return 0;
    return gemm_scales_off(M, K) + align_up((size_t)w8_rblocks(M) * 64, 256);
}

extern "C" int milo_w8a8_gemm(const milo_half* X, int64_t M, int64_t N, int64_t K, const void* w8, unsigned flags, milo_half* Y,
                              void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !w8 || !Y) return MILO_ERR_NULL;
    if (M < 1 || !w8_shape_ok(N, K) || !w8_shape_ok(M, K) || (flags & ~MILO_ACT_BF16)) return MILO_ERR_SHAPE;
    if (!workspace || workspace_bytes < milo_w8a8_gemm_workspace(M, N, K)) return MILO_ERR_WORKSPACE;
    if (!aligned16(X) || !aligned16(w8) || !aligned16(Y) || !aligned16(workspace)) return MILO_ERR_ALIGN;
    const bool bf = (flags & MILO_ACT_BF16) != 0;
    W8QuantArgs q;
    q.in = X;
    q.rows = M;
    q.K = K;
    q.codes = reinterpret_cast<uint8_t*>(workspace);
    q.scales = reinterpret_cast<float*>(q.codes + gemm_scales_off(M, K));
    q.blocked = 1;
    int st = launch_w8_quant(q, bf ? W8_BF16 : W8_F16, (hipStream_t)stream);
    if (st != MILO_OK) return st;
    if (M <= 16) {
        const dim3 grid((unsigned)w8_rblocks(N)), block(kStreamWaves * 64);
        if (bf) w8_stream_kernel<true><<<grid, block, 0, (hipStream_t)stream>>>(q.codes, q.scales, M, N, K, (const uint8_t*)w8, Y);
        else w8_stream_kernel<false><<<grid, block, 0, (hipStream_t)stream>>>(q.codes, q.scales, M, N, K, (const uint8_t*)w8, Y);
        return launch_status();
    }
    W8TileArgs a = {};
    a.A = q.codes;
    a.a_bytes = (uint64_t)w8_code_bytes(M, K);
    a.a_scales = q.scales;
    a.M = M;
    a.N = N;
    a.K = K;
    a.w = w8;
    a.out = Y;
    a.act_bf16 = bf;
    return launch_w8_tile(a, 0, M > 128 ? 256 : 128, (hipStream_t)stream);
}
