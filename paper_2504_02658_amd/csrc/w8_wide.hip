// The 8-bit product of small problems: few rows, or few tiles.
//
// A workgroup owns TM blocks of 16 rows by RN blocks of 16 output features over the whole K; its eight waves share K (integer sums:
// the split changes nothing) and every wave holds the whole tile's sums.  Operands go from memory to the matrix cores'
// registers as they are stored, without LDS and without a barrier in the loop, the next step's on their way while one is multiplied: a K
// loop through LDS takes a quarter of a microsecond per 64 columns whatever it multiplies there, when a compute unit has one
// workgroup.  What bounds it is the weight's bytes while there is one tile of rows, then the 64 bytes per cycle that a compute unit
// gets from its cache: (TM + RN) KB per 64 columns for TM RN matrix instructions.
//
// STAGED: up to 16 rows of a linear in their 16-bit type, which every workgroup quantizes for itself into LDS while its first fragments are
// on their way; so such a call is one launch.
#include "milo_host.h"
#include "w8_kernels.h"

namespace milo {

constexpr int kWideWaves = 8;

template <int TM, int RN, int EPI, bool BF, bool STAGED>
__global__ __launch_bounds__(kWideWaves * 64, 2) void w8_wide_kernel(const W8TileArgs a) {
    constexpr int NW = kWideWaves, B = TM + RN <= 2 ? 4 : TM + RN <= 4 ? 2 : 1;      // units (of 64 columns) of a step
    constexpr int OUTN = 16 * (EPI == 1 ? RN / 2 : RN);
    static_assert(EPI != 1 || RN % 2 == 0, "gate and up");
    static_assert(!STAGED || (EPI == 0 && TM == 1), "rows of a linear");
    constexpr int IN = BF ? W8_BF16 : W8_F16;
    __shared__ uint32_t s_top[STAGED ? 16 : 1][NW];
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    i32x4* const s_part = reinterpret_cast<i32x4*>(smem);           // [wave][tile][lane]
    unsigned char* const codes = smem + NW * TM * RN * 1024;        // STAGED: piece c of 16 columns of row m at (c * rows + m) * 16
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int m16 = lane & 15, c16 = lane >> 4;
    const int kb = (int)w8_kblocks(a.K);
    int mt, nt;
    w8_tile_of(blockIdx.x, a.m_tiles, a.n_tiles, a.group_m, a.span, &mt, &nt);
    const int64_t n0 = (int64_t)nt * OUTN;
    int64_t row0;
    int rows;
    const void *w0, *w1;
    if constexpr (EPI == 0) {
        row0 = (int64_t)mt * (TM * 16);
        rows = (int)(a.M - row0 < TM * 16 ? a.M - row0 : TM * 16);
        w0 = w1 = a.w;
    } else {
        const TileDesc t = a.tiles[mt];
        row0 = t.row0;
        rows = t.rows;
        if (rows == 0) return;
        const milo_w8_expert& e = a.experts[t.expert];
        w0 = EPI == 1 ? e.w1 : e.w2;
        w1 = EPI == 1 ? e.w3 : e.w2;
    }
    const int nblocks = (int)w8_rblocks(a.N);
    GlobalFrag wp[RN], xp[TM];
#pragma unroll
    for (int n = 0; n < RN; ++n) {
        const int b = (int)(n0 >> 4) + (EPI == 1 ? n % (RN / 2) : n), bb = b < nblocks ? b : nblocks - 1;
        wp[n] = global_frag(reinterpret_cast<const char*>(EPI == 1 && n >= RN / 2 ? w1 : w0) + (int64_t)bb * kb * 1024) + lane;
    }
#pragma unroll
    for (int m = 0; m < TM; ++m) {
        if constexpr (EPI == 0) {
            const int64_t b = (row0 >> 4) + m, last = w8_rblocks(a.M) - 1;
            xp[m] = global_frag(a.A + (b < last ? b : last) * kb * 1024) + lane;
        } else {
            int64_t r = m * 16 + m16;
            r = row0 + (r < rows ? r : 0);
            if (EPI == 1) r = a.x_rows[r];
            xp[m] = global_frag(a.A + r * kb * 64) + c16;
        }
    }
    constexpr int XSTEP = EPI == 0 ? 64 : 4;                        // pieces of 16 bytes from a unit to the next
    u32x4 wf[2][B][RN], xf[2][B][TM];
    auto fetch = [&](int u, int to) {
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int v = u + i < kb ? u + i : kb - 1;
#pragma unroll
            for (int n = 0; n < RN; ++n) wf[to][i][n] = wp[n][v * 64];
            if constexpr (!STAGED) {
#pragma unroll
                for (int m = 0; m < TM; ++m) xf[to][i][m] = xp[m][v * XSTEP];
            }
        }
    };
    i32x4 acc[TM][RN];
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
        for (int n = 0; n < RN; ++n) acc[m][n] = i32x4{0, 0, 0, 0};
    auto work = [&](int u, int from) {
        if constexpr (STAGED) {
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const int v = u + i < kb ? u + i : kb - 1;
                xf[from][i][0] = u32x4{0u, 0u, 0u, 0u};
                if (m16 < rows) xf[from][i][0] = *reinterpret_cast<const u32x4*>(codes + ((v * 4 + c16) * rows + m16) * 16);
            }
        }
        fetch(u + B * NW, from ^ 1);
        asm volatile("" ::: "memory");              // (the loads stay in front)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            if (B > 1 && u + i >= kb) break;
#pragma unroll
            for (int m = 0; m < TM; ++m)
#pragma unroll
                for (int n = 0; n < RN; ++n) acc[m][n] = mfma16_i8(wf[from][i][n], xf[from][i][m], acc[m][n]);
        }
    };
    if (wave * B < kb) fetch(wave * B, 0);
    if constexpr (STAGED) {
        // up to eight waves share a row
        const int share = rows > 4 ? 1 : rows > 2 ? 2 : rows > 1 ? 4 : 8, part = wave % share, pieces = kb * 4;
        const char* const X = reinterpret_cast<const char*>(a.A);
        for (int m = wave / share; m < rows; m += NW / share) {
            uint32_t top = 0u;
            for (int p = part * 64 + lane; p < pieces; p += share * 64) top = raw_top<IN>(load16<IN>(X + m * a.K * 2, (int64_t)p * 16, a.K), top);
            top = wave_max(top_bits<IN>(top));
            if (lane == 0) s_top[m][part] = top;
        }
        __syncthreads();
        for (int m = wave / share; m < rows; m += NW / share) {
            uint32_t top = s_top[m][0];
            for (int i = 1; i < share; ++i) top = s_top[m][i] > top ? s_top[m][i] : top;
            const RowStep st = row_step(top);
            for (int p = part * 64 + lane; p < pieces; p += share * 64) {
                float v[16];
                raw_values<IN>(load16<IN>(X + m * a.K * 2, (int64_t)p * 16, a.K), v);
                *reinterpret_cast<u32x4*>(codes + (p * rows + m) * 16) = row_codes16(v, st);
            }
        }
        __syncthreads();
    }
    for (int u = wave * B; u < kb; u += 2 * B * NW) {
        work(u, 0);
        if (u + B * NW >= kb) break;
        work(u + B * NW, 1);
    }
#pragma unroll
    for (int m = 0; m < TM; ++m)
#pragma unroll
        for (int n = 0; n < RN; ++n) s_part[(wave * TM * RN + m * RN + n) * 64 + lane] = acc[m][n];
    __syncthreads();
    // Sums over the waves and output: a wave takes every eighth tile of 16 x 16 (gate and up: their pair)
    auto total = [&](int tile) {
        i32x4 s = s_part[tile * 64 + lane];
#pragma unroll
        for (int w = 1; w < NW; ++w) s += s_part[(w * TM * RN + tile) * 64 + lane];
        return s;
    };
    constexpr int ON = OUTN / 16;
    const bool vec = (a.N & 3) == 0;
    const auto sw0 = global_float(w8_scales(w0, a.N, a.K)), sw1 = global_float(w8_scales(w1, a.N, a.K));
    for (int t = wave; t < TM * ON; t += NW) {
        const int m = t / ON, n = t - m * ON, r = m * 16 + m16;
        const int64_t col = n0 + n * 16 + c16 * 4;
        const i32x4 s = total(m * RN + n);
        i32x4 s1 = s;
        if constexpr (EPI == 1) s1 = total(m * RN + n + RN / 2);
        if (r >= rows || col >= a.N) continue;
        const int64_t row = row0 + r;
        const int left = (int)(a.N - col < 4 ? a.N - col : 4);
        int64_t to = row;
        float sx;
        if constexpr (STAGED) {
            const int share = rows > 4 ? 1 : rows > 2 ? 2 : rows > 1 ? 4 : 8;
            uint32_t top = s_top[r][0];
            for (int i = 1; i < share; ++i) top = s_top[r][i] > top ? s_top[r][i] : top;
            sx = row_step(top).s;
        } else if constexpr (EPI == 0) sx = a.a_scales[row];
        else if constexpr (EPI == 1) sx = a.a_scales[a.x_rows[row]];
        else {
            to = a.x_rows[row];
            sx = a.a_scales[row] * a.gates[to];
        }
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = (float)s[j] * sx * sw0[col + j];
            if constexpr (EPI == 1) v[j] = silu_times(v[j], (float)s1[j] * sx * sw1[col + j]);
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

template <int TM, int RN, int EPI, bool BF, bool STAGED = false>
static int launch_wide(W8TileArgs a, hipStream_t stream) {
    constexpr int OUTN = 16 * (EPI == 1 ? RN / 2 : RN), most = kWideWaves * TM * RN * 1024 + (STAGED ? kW8WideStaged : 0);
    const int lds = kWideWaves * TM * RN * 1024 + (STAGED ? (int)(a.M * w8_kblocks(a.K) * 64) : 0);
    if constexpr (most > 64 * 1024) {
        static bool raised[64] = {false};
        const int st = raise_lds(reinterpret_cast<const void*>(w8_wide_kernel<TM, RN, EPI, BF, STAGED>), most, raised);
        if (st != MILO_OK) return st;
    }
    if (EPI == 0) a.m_tiles = (int)((a.M + TM * 16 - 1) / (TM * 16));
    a.n_tiles = (int)((a.N + OUTN - 1) / OUTN);
    static_assert(kWideWaves == 8, "512 threads");
    if ((int64_t)a.m_tiles * a.n_tiles > kW8MaxGroups) return MILO_ERR_SHAPE;
    w8_wide_kernel<TM, RN, EPI, BF, STAGED><<<dim3((unsigned)(a.m_tiles * a.n_tiles)), dim3(kWideWaves * 64), lds, stream>>>(a);
    return launch_status();
}
template <bool BF>
static int launch_wide_linear(const W8TileArgs& a, int tm, int rn, hipStream_t stream) {
    if (tm == 4) return launch_wide<4, 4, 0, BF>(a, stream);
    if (tm == 2) return rn == 4 ? launch_wide<2, 4, 0, BF>(a, stream) : launch_wide<2, 2, 0, BF>(a, stream);
    if (rn == 4) return launch_wide<1, 4, 0, BF>(a, stream);
    return rn == 2 ? launch_wide<1, 2, 0, BF>(a, stream) : launch_wide<1, 1, 0, BF>(a, stream);
}
template <bool BF>
static int launch_staged(const W8TileArgs& a, W8Kernel k, hipStream_t stream) {
    if (k == W8_WIDE_16x64) return launch_wide<1, 4, 0, BF, true>(a, stream);
    if (k == W8_WIDE_16x32) return launch_wide<1, 2, 0, BF, true>(a, stream);
    return launch_wide<1, 1, 0, BF, true>(a, stream);
}
int launch_w8_staged(const W8TileArgs& a, W8Kernel k, hipStream_t stream) {
    return a.act_bf16 ? launch_staged<true>(a, k, stream) : launch_staged<false>(a, k, stream);
}
int launch_w8_wide(const W8TileArgs& a, int epi, int tm, int rn, hipStream_t stream) {
    if (epi == 0) return a.act_bf16 ? launch_wide_linear<true>(a, tm, rn, stream) : launch_wide_linear<false>(a, tm, rn, stream);
    if (tm != 2 || rn != 4) return MILO_ERR_SHAPE;          // (experts: this shape alone)
    return epi == 1 ? launch_wide<2, 4, 1, false>(a, stream) : launch_wide<2, 4, 2, false>(a, stream);
}

}  // namespace milo
