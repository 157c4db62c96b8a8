// Linears in 8-bit integers: milo_pack_w8, milo_w8a8_gemm and the tiled product that the MoE layer shares.
#include <math.h>

#include <type_traits>

#include "milo_host.h"
#include "w8_kernels.h"

namespace milo {

// A row's sums have to fit 32 bits: 127 * 127 * K < 2^31.
constexpr int64_t kW8MaxK = 1 << 17;

// (and the quantizer's grid of up to 1024 threads per row fits 32 bits of work items: 2^22 rows go with K <= 16384, where it takes 256)
bool w8_shape_ok(int64_t N, int64_t K) {
    return N >= 1 && K >= 1 && K <= kW8MaxK && N < (int64_t(1) << 22) && N <= (int64_t(1) << 36) / K;
}
// (and a grid's work items fit 32 bits: one per 16 outputs with the smallest tiles that large products take)
static bool w8_linear_ok(int64_t M, int64_t N, int64_t K) { return w8_shape_ok(N, K) && w8_shape_ok(M, K) && M <= (int64_t(1) << 36) / N; }

// ---------------------------------------------------------------------------------------------
// Row quantizer: a row is read once for its largest magnitude and, while it fits the registers of its TPR threads,
// quantized from there.
// (HELD: pieces of 16 that a thread holds.)
template <int IN, int TPR, int ROWS, int HELD, bool BLOCKED>
__global__ __launch_bounds__(TPR * ROWS) void w8_quant_kernel(const W8QuantArgs a, int kb) {
    constexpr int SZ = IN == W8_F32 ? 4 : 2;
    __shared__ uint32_t s_top[TPR * ROWS / 64];
    const int tid = threadIdx.x % TPR, of = threadIdx.x / TPR;
    const int64_t row = (int64_t)blockIdx.x * ROWS + of;
    const bool there = row < a.rows;
    const char* in = reinterpret_cast<const char*>(a.in) + (there ? row : 0) * a.K * SZ;
    const int64_t K = there ? a.K : 0;          // (rows beyond the last are all zero)
    const int pieces = kb * 4;                  // of 16 columns, with the padding
    W8Raw<IN> held[HELD];
    uint32_t top = 0u;
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int p = tid + i * TPR;
        held[i] = W8Raw<IN>{};
        if (p < pieces) held[i] = load16<IN>(in, (int64_t)p * 16, K);
    }
#pragma unroll
    for (int i = 0; i < HELD; ++i) top = raw_top<IN>(held[i], top);
    for (int p = tid + HELD * TPR; p < pieces; p += TPR) top = raw_top<IN>(load16<IN>(in, (int64_t)p * 16, K), top);
    top = wave_max(top_bits<IN>(top));
    if constexpr (TPR > 64) {
        if ((threadIdx.x & 63) == 0) s_top[threadIdx.x >> 6] = top;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < TPR / 64; ++w) {
            const uint32_t o = s_top[of * (TPR / 64) + w];
            top = o > top ? o : top;
        }
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
    for (int i = 0; i < HELD; ++i)
        if (tid + i * TPR < pieces) put(tid + i * TPR, held[i]);
    for (int p = tid + HELD * TPR; p < pieces; p += TPR) put(p, load16<IN>(in, (int64_t)p * 16, K));
    if (tid == 0) a.scales[row] = st.s;
}

template <int IN, bool BLOCKED>
static int launch_quant(const W8QuantArgs& a, hipStream_t stream) {
    const int kb = (int)w8_kblocks(a.K);
    const int64_t rows = BLOCKED ? w8_rblocks(a.rows) * 16 : a.rows;
    if (rows == 0) return MILO_OK;
    // Few rows: as many threads as a row has pieces (128 rows of 4096: 5.8 us against 8.0 with a wave per row).  Many rows: 1024 threads on
    // as many rows as they can hold, so that the rows of a block leave one compute unit together.
    auto launch = [&](auto kernel, int threads, int per) { kernel<<<dim3((unsigned)((rows + per - 1) / per)), dim3(threads), 0, stream>>>(a, kb); };
    const int pieces = kb * 4;
    if (rows < 1024) {
        if (pieces <= 256) launch(w8_quant_kernel<IN, 256, 1, 1, BLOCKED>, 256, 1);
        else if (pieces <= 1024) launch(w8_quant_kernel<IN, 1024, 1, 1, BLOCKED>, 1024, 1);
        else launch(w8_quant_kernel<IN, 1024, 1, 4, BLOCKED>, 1024, 1);
    } else {
        if (pieces <= 256) launch(w8_quant_kernel<IN, 64, 16, 4, BLOCKED>, 1024, 16);
        else if (pieces <= 1024) launch(w8_quant_kernel<IN, 256, 4, 4, BLOCKED>, 1024, 4);
        else launch(w8_quant_kernel<IN, 1024, 1, 4, BLOCKED>, 1024, 1);
    }
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

// The tiled product.  WM x WN waves (times WK, which share K), each with TM x TN tiles of 32 x 32; NS stages of 64 columns in LDS.
// Copies go from memory to LDS directly, as the operands are stored.  What a stage of the widest tile costs: 16 KB + 8 KB from the L2,
// 8 matrix instructions of 32 cycles per wave, two of its workgroups per compute unit.  4096 x 4096 x 14336: 213 us on a cool card with the matrix
// cores busy 70 % of the cycles at 1.55 GHz, 236 back to back: the clock falls under this load.  Small tiles are bound by the L2 (about 11 to 14 TB/s into LDS in all), so the widest that fills the chip is taken.
template <int WM, int WN, int WK, int TM, int TN, int NS, int EPI, bool BF>
__global__ __launch_bounds__(WM * WN * WK * 64, 2) void w8_tile_kernel(const W8TileArgs a) {
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32, NW = WM * WN;
    constexpr int ABLK = BM / 16, BBLK = BN / 16;       // 1-KB blocks of 64 columns
    constexpr int PA = ABLK / NW, PB = BBLK / NW;       // of them, copied by one wave
    constexpr int PART = (ABLK + BBLK) * 1024, STAGE = WK * PART;
    constexpr int OUTN = EPI == 1 ? BN / 2 : BN;        // output columns of a tile
    static_assert(ABLK % NW == 0 && (EPI == 1 ? BBLK / 2 : BBLK) % NW == 0, "every wave copies as many blocks");
    static_assert(WK == 1 || WK == 2, "an even number of blocks of 64 columns");
    static_assert(WK == 1 || NS * STAGE >= NW * TM * TN * 4096, "room for the second half's sums");
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int lane = threadIdx.x & 63, wave_all = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int wk = wave_all / NW, wave = wave_all - wk * NW;
    const int kb = (int)w8_kblocks(a.K), stages = kb / WK;
    int mt, nt;
    w8_tile_of(blockIdx.x, a.m_tiles, a.n_tiles, a.group_m, a.span, &mt, &nt);
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
    // EPI 1, 2: four neighbouring lanes copy the 64 bytes of one row, so that they make one request (a lane per row, in the blocks' order, makes four: 512
    // tokens of 8 experts of 14336 x 4096 497 us against 483).  Then rows are 64 bytes apart in LDS, and of 16 rows that are read at once
    // four would meet in the same banks: piece p of row r is put at p ^ (r / 4 % 4).
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
            aoff[i] = (uint32_t)(b * kb + wk) * 1024u + lane * 16;
        } else {
            int r = b * 16 + (lane >> 2);
            r = (int)row0 + (r < rows ? r : 0);         // (rows beyond the tile's: computed, not stored)
            const int64_t src = EPI == 1 ? a.x_rows[r] : r;
            aoff[i] = (uint32_t)(src * kb * 64) + wk * 64 + ((lane ^ lane >> 4) & 3) * 16;
        }
    }
#pragma unroll
    for (int i = 0; i < PB; ++i) boff[i] = (uint32_t)(((wave + i * NW) % (OUTN / 16)) * kb + wk) * 1024u + lane * 16;
    auto issue = [&](int c) {
        unsigned char* const to = smem + (c % NS) * STAGE + wk * PART + wave * 1024;
#pragma unroll
        for (int i = 0; i < PA; ++i) {
            const uint32_t o = aoff[i];
            __builtin_amdgcn_raw_ptr_buffer_load_lds(ra, (LdsDst)(to + i * NW * 1024), 16, o, 0, 0, 0);
            aoff[i] += (EPI == 0 ? 1024u : 64u) * WK;
        }
#pragma unroll
        for (int i = 0; i < PB; ++i) {
            const uint32_t o = boff[i];
            if (EPI == 1 && i >= PB / 2) __builtin_amdgcn_raw_ptr_buffer_load_lds(rb1, (LdsDst)(to + (ABLK + i * NW) * 1024), 16, o, 0, 0, 0);
            else __builtin_amdgcn_raw_ptr_buffer_load_lds(rb0, (LdsDst)(to + (ABLK + i * NW) * 1024), 16, o, 0, 0, 0);
            boff[i] += 1024u * WK;
        }
    };
    const int wm = wave % WM, wn = wave / WM, l32 = lane & 31, h = lane >> 5;
    const int frag = (l32 >> 4) * 1024 + h * 256 + (l32 & 15) * 16;
    const int afrag = EPI == 0 ? frag : (l32 >> 4) * 1024 + (l32 & 15) * 64 + ((h ^ l32 >> 2) & 3) * 16;
    // The wave's m-th block of 32 rows is block m * WM + wm of the tile; blocks past the tile's rows take no part (the loop is there
    // once for every number of blocks, and its body has no branches).
    const int blocks = (rows + 31) / 32, used = (blocks - wm + WM - 1) / WM;
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
    auto k_loop = [&](auto mbu) {
        constexpr int MBU = decltype(mbu)::value;
        u32x4 af[2][MBU > 0 ? MBU : 1], bf[2][TN];
        auto read = [&](int c, int k) {
            const unsigned char* const as = smem + (c % NS) * STAGE + wk * PART + wm * 2048 + (EPI == 0 ? frag + k * 512 : afrag ^ k * 32);
            const unsigned char* const bs = smem + (c % NS) * STAGE + wk * PART + ABLK * 1024 + frag + k * 512;
            if constexpr (MBU > 0) {
#pragma unroll
                for (int n = 0; n < TN; ++n) bf[k][n] = *reinterpret_cast<const u32x4*>(bs + brow(n) * 2048);
#pragma unroll
                for (int m = 0; m < MBU; ++m) af[k][m] = *reinterpret_cast<const u32x4*>(as + m * WM * 2048);
            }
        };
        auto multiply = [&](int k) {
#pragma unroll
            for (int m = 0; m < MBU; ++m)
#pragma unroll
                for (int n = 0; n < TN; ++n) acc[n][m] = mfma32_i8(bf[k][n], af[k][m], acc[n][m]);
        };
        // one LDS read behind each of the first matrix instructions, instead of all of them in front
        auto mix = [&] {
            if constexpr (MBU * TN >= MBU + TN) {
#pragma unroll
                for (int i = 0; i < MBU + TN; ++i) {
                    __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
                }
                __builtin_amdgcn_sched_group_barrier(0x8, MBU * TN - MBU - TN, 0);
            }
            __builtin_amdgcn_sched_barrier(0);
        };
        auto arrive = [&](auto counted, bool all) {
            if (!decltype(counted)::value && all) wait_vmem();
            else MILO_WAIT_VMEM((NS - 2) * (PA + PB));
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
        };
        for (int c = 0; c < NS - 1 && c < stages; ++c) issue(c);
        arrive(std::bool_constant<false>{}, stages < NS - 1);
        if (NS - 1 < stages) issue(NS - 1);
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
        for (; c + NS < stages; ++c) stage(std::bool_constant<true>{});
        for (; c < stages; ++c) stage(std::bool_constant<false>{});
    };
    static_assert(TM <= 2, "a loop for every number of blocks");
    if (TM >= 2 && used >= 2) k_loop(std::integral_constant<int, TM >= 2 ? 2 : 1>{});
    else if (used >= 1) k_loop(std::integral_constant<int, 1>{});
    else k_loop(std::integral_constant<int, 0>{});          // (copies its share, and keeps the barriers)
    if constexpr (WK == 2) {
        // the waves of the odd blocks hand their sums to those of the even ones, through the stages that nobody reads any more
        i32x4* const part = reinterpret_cast<i32x4*>(smem) + wave * (TM * TN * 256) + lane;
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __syncthreads();
        if (wk == 1) {
#pragma unroll
            for (int n = 0; n < TN; ++n)
#pragma unroll
                for (int m = 0; m < TM; ++m)
#pragma unroll
                    for (int i = 0; i < 4; ++i) part[((n * TM + m) * 4 + i) * 64] = i32x4{acc[n][m][4 * i], acc[n][m][4 * i + 1], acc[n][m][4 * i + 2], acc[n][m][4 * i + 3]};
        }
        __syncthreads();
#pragma unroll
        for (int n = 0; n < TN; ++n)
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const i32x4 v = part[((n * TM + m) * 4 + i) * 64];
#pragma unroll
                    for (int j = 0; j < 4; ++j) acc[n][m][4 * i + j] += v[j];
                }
    }
    // Output.  A lane has features 8 i + 4 h + 0..3 of row l32 (of 32): stored from there, an instruction would touch 64 lines.  So the tile goes
    // through LDS, which nobody reads any more, and leaves it by whole rows.
    const auto sw0 = global_float(w8_scales(w0, a.N, a.K)), sw1 = global_float(w8_scales(w1, a.N, a.K));
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __syncthreads();
    // of the wave's m-th block: put(row of the tile, column of the tile, four values)
    auto block = [&](int m, auto&& put) {
        const int r = (m * WM + wm) * 32 + l32;
        if (r >= rows || wk != 0) return;           // (with K in two halves, the first one's waves have the sums)
        const int64_t row = row0 + r;
        float sx;
        if constexpr (EPI == 0) sx = a.a_scales[row];
        else if constexpr (EPI == 1) sx = a.a_scales[a.x_rows[row]];
        else sx = a.a_scales[row] * a.gates[a.x_rows[row]];
#pragma unroll
        for (int n = 0; n < (EPI == 1 ? TN / 2 : TN); ++n)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int c = (EPI == 1 ? wn * (TN / 2) + n : wn * TN + n) * 32 + 8 * i + 4 * h;
                float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                if (n0 + c < a.N) {         // (there are scales for whole blocks of 16)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        v[j] = (float)acc[n][m][4 * i + j] * sx * sw0[n0 + c + j];
                        if constexpr (EPI == 1) v[j] = silu_times(v[j], (float)acc[n + TN / 2][m][4 * i + j] * sx * sw1[n0 + c + j]);
                    }
                }
                put(r, c, v);
            }
    };
    auto each = [&](auto&& put) {
#pragma unroll
        for (int m = 0; m < TM; ++m) block(m, put);
    };
    constexpr int threads = WM * WN * WK * 64;
    const int tid = threadIdx.x;
    if constexpr (EPI != 0) {
        // fp32.  SwiGLU rows: the quantizer that follows has to see the value that it rounds.  (16-bit fixed point with a scale per row and 128
        // features moves one code in 600, and one step of a code in 600 is 0.16 % of the layer's output, eight times what fp16 rounds off; it took
        // 35 us less of 540, 4096 tokens of 66 experts of 1408.)  A pair's weighted output: the sum over a token's pairs may cancel, and may
        // fit 16 bits where a term does not.  The room is that of all rows of half as many columns (gate and up), or of WM blocks of rows.
        float* const tile = reinterpret_cast<float*>(smem);
        constexpr int PITCH = OUTN + 4, Q = OUTN / 4, PARTS = EPI == 1 ? 1 : TM, ROWS = BM / PARTS;
        static_assert(ROWS * PITCH * 4 <= NS * STAGE, "room for a part of the tile");
        auto put = [&](int r, int c, const float (&v)[4]) { *reinterpret_cast<f32x4*>(tile + (r % ROWS) * PITCH + c) = f32x4{v[0], v[1], v[2], v[3]}; };
#pragma unroll
        for (int part = 0; part < PARTS; ++part) {
            if (part > 0) __syncthreads();              // (the part before has left)
            if constexpr (PARTS == 1) each(put);
            else block(part, put);
            __syncthreads();
            for (int r = part * ROWS + tid / Q; r < rows && r < (part + 1) * ROWS; r += threads / Q) {
                const int c = (tid % Q) * 4;
                const f32x4 v = *reinterpret_cast<const f32x4*>(tile + (r % ROWS) * PITCH + c);
                float* const to = reinterpret_cast<float*>(a.out) + (EPI == 1 ? row0 + r : (int64_t)a.x_rows[row0 + r]) * a.N + n0 + c;
                if ((a.N & 3) == 0) {
                    if (n0 + c < a.N) *reinterpret_cast<f32x4*>(to) = v;
                } else {
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        if (n0 + c + j < a.N) to[j] = v[j];
                }
            }
        }
    } else if ((a.N & 7) != 0) {
        const bool vec = (a.N & 3) == 0;
        each([&](int r, int c, const float (&v)[4]) {
            const int64_t col = n0 + c;
            if (col >= a.N) return;
            store4<BF>(reinterpret_cast<uint16_t*>(a.out) + (row0 + r) * a.N + col, v, (int)(a.N - col < 4 ? a.N - col : 4), vec);
        });
    } else {
        uint16_t* const tile = reinterpret_cast<uint16_t*>(smem);
        constexpr int PITCH = BN + 8;
        static_assert(BM * PITCH * 2 <= NS * STAGE, "room for the tile");
        each([&](int r, int c, const float (&v)[4]) { store4<BF>(tile + r * PITCH + c, v, 4, true); });
        __syncthreads();
        for (int r = tid / (BN / 8); r < rows; r += threads / (BN / 8)) {
            const int c = (tid % (BN / 8)) * 8;
            if (n0 + c >= a.N) continue;
            *reinterpret_cast<u32x4*>(reinterpret_cast<uint16_t*>(a.out) + (row0 + r) * a.N + n0 + c) = *reinterpret_cast<const u32x4*>(tile + r * PITCH + c);
        }
    }
}

template <int WM, int WN, int WK, int TM, int TN, int NS, int EPI, bool BF>
static int launch_tile(W8TileArgs a, hipStream_t stream) {
    constexpr int BM = WM * TM * 32, BN = WN * TN * 32, OUTN = EPI == 1 ? BN / 2 : BN, lds = NS * WK * (BM + BN) * 64;
    if constexpr (lds > 64 * 1024) {
        static bool raised[64] = {false};
        const int st = raise_lds(reinterpret_cast<const void*>(w8_tile_kernel<WM, WN, WK, TM, TN, NS, EPI, BF>), lds, raised);
        if (st != MILO_OK) return st;
    }
    if (EPI == 0) a.m_tiles = (int)((a.M + BM - 1) / BM);
    a.n_tiles = (int)((a.N + OUTN - 1) / OUTN);
    static_assert(WM * WN * WK <= 8, "512 threads");
    if ((int64_t)a.m_tiles * a.n_tiles > kW8MaxGroups) return MILO_ERR_SHAPE;
    w8_tile_kernel<WM, WN, WK, TM, TN, NS, EPI, BF><<<dim3((unsigned)(a.m_tiles * a.n_tiles)), dim3(WM * WN * WK * 64), lds, stream>>>(a);
    return launch_status();
}
template <bool BF>
static int launch_linear_tile(const W8TileArgs& a, W8Kernel k, hipStream_t stream) {
    switch (k) {
        case W8_TILE_64x128: return launch_tile<2, 2, 2, 1, 2, 4, 0, BF>(a, stream);
        case W8_TILE_128x128: return launch_tile<2, 2, 1, 2, 2, 4, 0, BF>(a, stream);
        default: return launch_tile<2, 4, 1, 2, 2, 3, 0, BF>(a, stream);        // (72 KB of LDS: two workgroups share a compute unit)
    }
}
static int launch_w8_tile(const W8TileArgs& a, int epi, W8Kernel k, hipStream_t stream) {
    if (epi == 0) return a.act_bf16 ? launch_linear_tile<true>(a, k, stream) : launch_linear_tile<false>(a, k, stream);
    if (k != W8_TILE_128x256) return MILO_ERR_SHAPE;        // (experts: these rows alone)
    if (epi == 1) return launch_tile<2, 4, 1, 2, 2, 3, 1, false>(a, stream);
    // Tiles that are half as wide where the wide ones would leave half of the compute units without one.  The layer, us: 45 tokens of 17 experts of
    // 2730 x 1000, 76 wide tiles, 50.8 against 55.6; 512 of 8 of 4096 x 2048, 128 of them, 80 against 90; where they fill the chip they cost
    // more: 512 of 8 of 14336 x 4096, 256 of them, 451 against 419.
    if ((int64_t)a.m_tiles * ((a.N + 255) / 256) <= device_cus() / 2)
        return launch_tile<2, 4, 1, 2, 1, 4, 2, false>(a, stream);
    return launch_tile<2, 4, 1, 2, 2, 3, 2, false>(a, stream);
}
int launch_w8_product(const W8TileArgs& a, int epi, W8Kernel k, hipStream_t stream) {
    switch (k) {
        case W8_WIDE_16x16: return launch_w8_wide(a, epi, 1, 1, stream);
        case W8_WIDE_16x32: return launch_w8_wide(a, epi, 1, 2, stream);
        case W8_WIDE_16x64: return launch_w8_wide(a, epi, 1, 4, stream);
        case W8_WIDE_32x32: return launch_w8_wide(a, epi, 2, 2, stream);
        case W8_WIDE_32x64: return launch_w8_wide(a, epi, 2, 4, stream);
        case W8_WIDE_64x64: return launch_w8_wide(a, epi, 4, 4, stream);
        default: return launch_w8_tile(a, epi, k, stream);
    }
}

// The kernel of a linear.  Up to 16 rows every weight byte is read once, and what counts is that all compute units read: as many features
// per workgroup as leave at least 192 workgroups (16 rows, N = 14336, K = 4096: 20.4, 18.8, 18.2 us with 16, 32, 64 features; N = 4096,
// K = 14336: 20.3, 24.2, 31.4).  More rows: the least of the estimates
//     base + blocks of 64 columns * (lat + step * max(rounds, full * workgroups per compute unit))
// with rounds = 1 for the kernels whose workgroups share a compute unit, else the workgroups per compute unit rounded up, and the constants
// (us, at 256 compute units) fitted to 2520 times of 180 shapes, 1 to 4096 rows, N and K from 512 to 14336, in every kernel.  The
// choice costs 3.5 % against the best of 14 kernels of each shape on average, 25 % at worst (96 x 8192 x 8192); 32 x 64 or 256 x 256,
// whichever is better, would cost 13 %.  (Tiles of 256 x 256 are gone: with their 128 KB of LDS a compute unit has one workgroup and nothing to do
// in its epilogue; 4096 x 2048 x 1408 41.4 us against 33.7, 4096 x 14336 x 4096 298 against 296, 4096 x 4096 x 14336 257 against 265.)
W8Kernel w8_linear_kernel(int64_t M, int64_t N, int64_t K) {
    if (M <= 16) return N >= 192 * 64 ? W8_WIDE_16x64 : N >= 192 * 32 ? W8_WIDE_16x32 : W8_WIDE_16x16;
    struct Cost {
        W8Kernel kernel;
        int rows, cols;
        bool whole;         // whole rounds
        double base, lat, step, full;
    };
    static const Cost costs[] = {
        {W8_WIDE_16x32, 16, 32, false, 7.91, 0.0235, 0.0118, 3.56}, {W8_WIDE_32x32, 32, 32, false, 8.16, 0.0243, 0.0378, 1.60},
        {W8_WIDE_32x64, 32, 64, false, 8.71, 0.0474, 0.0056, 13.9}, {W8_WIDE_64x64, 64, 64, false, 9.51, 0.0158, 0.0882, 1.64},
        {W8_TILE_64x128, 64, 128, true, 8.76, 0.0, 0.240, 1.24},    {W8_TILE_128x128, 128, 128, true, 13.7, 0.0218, 0.235, 1.26},
        {W8_TILE_128x256, 128, 256, true, 12.7, 0.0, 0.456, 1.25}};
    W8Kernel best = W8_TILE_128x256;
    double least = 0.0;
    const double kb = (double)w8_kblocks(K), cus = device_cus();
    for (const Cost& c : costs) {
        const double groups = (double)((M + c.rows - 1) / c.rows) * (double)((N + c.cols - 1) / c.cols) / cus;
        const double per = fmax(c.whole ? ceil(groups) : 1.0, c.full * groups);
        const double t = c.base + kb * (c.lat + c.step * per);
        if (least == 0.0 || t < least) {
            least = t;
            best = c.kernel;
        }
    }
    return best;
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
    if (!w8_linear_ok(M, N, K)) return 0;
    return gemm_scales_off(M, K) + align_up((size_t)w8_rblocks(M) * 64, 256);
}

extern "C" int milo_w8a8_gemm(const milo_half* X, int64_t M, int64_t N, int64_t K, const void* w8, unsigned flags, milo_half* Y,
                              void* workspace, size_t workspace_bytes, void* stream) {
    if (!X || !w8 || !Y) return MILO_ERR_NULL;
    if (!w8_linear_ok(M, N, K) || (flags & ~MILO_ACT_BF16)) return MILO_ERR_SHAPE;
    if (!workspace || workspace_bytes < milo_w8a8_gemm_workspace(M, N, K)) return MILO_ERR_WORKSPACE;
    if (!aligned16(X) || !aligned16(w8) || !aligned16(Y) || !aligned16(workspace)) return MILO_ERR_ALIGN;
    const bool bf = (flags & MILO_ACT_BF16) != 0;
    const W8Kernel kernel = w8_linear_kernel(M, N, K);
    W8TileArgs a = {};
    a.M = M;
    a.N = N;
    a.K = K;
    a.w = w8;
    a.group_m = 8;
    a.span = 1;
    a.out = Y;
    a.act_bf16 = bf;
    if (M <= 16 && M * w8_kblocks(K) * 64 <= kW8WideStaged) {
        a.A = reinterpret_cast<const uint8_t*>(X);
        return launch_w8_staged(a, kernel, (hipStream_t)stream);
    }
    W8QuantArgs q;
    q.in = X;
    q.rows = M;
    q.K = K;
    q.codes = reinterpret_cast<uint8_t*>(workspace);
    q.scales = reinterpret_cast<float*>(q.codes + gemm_scales_off(M, K));
    q.blocked = 1;
    const int st = launch_w8_quant(q, bf ? W8_BF16 : W8_F16, (hipStream_t)stream);
    if (st != MILO_OK) return st;
    a.A = q.codes;
    a.a_bytes = (uint64_t)w8_code_bytes(M, K);
    a.a_scales = q.scales;
    return launch_w8_product(a, 0, kernel, (hipStream_t)stream);
}

// For the tests: which kernel a linear takes (W8Kernel; for the current device, or without one for 256 compute units).
extern "C" int milo_w8a8_route(int64_t M, int64_t N, int64_t K) { return (int)w8_linear_kernel(M, N, K); }
