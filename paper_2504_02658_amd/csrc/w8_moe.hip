// milo_moe_w8a8_forward: top-k routed SwiGLU experts over 8-bit integer linears.
//
// Up to kFewTokens tokens, two products, both bound by the bytes of the weights of the experts that some token goes to:
//   few_up    a workgroup owns 16 of the F features of one expert (gate and up): it finds the expert's tokens in the ids,
//             multiplies their codes, and writes H = SiLU(gate) * up with the largest magnitude of its 16 features per row
//   few_down  a workgroup owns 16 of the H features of the output and walks all experts: it adds each expert's product,
//             weighted, to the tokens' sums, so that nothing is left to combine
// Either quantizes its rows itself while their codes are few (kFewUpStaged, kFewDownStaged), else a launch of the row quantizer goes
// in front of it: two to four launches.
// More tokens: the activations' rows are quantized once, pairs grouped per expert (route_kernel of moe.hip), gate and up as one
// grouped product over the tiles, the SwiGLU rows quantized, the grouped down projection, and the sum over a token's pairs.
#include "milo_host.h"
#include "w8_kernels.h"

namespace milo {

constexpr int kFewTokens = 16, kFewMaxPairs = 128;
constexpr int kFewUpThreads = 256, kFewDownThreads = 1024;

struct W8FewArgs {
    const void* X;
    int T, topk, E;
    int64_t H, F;
    const milo_w8_expert* experts;
    const int32_t* ids;
    const float* gates;
    int32_t* status;        // routing status
    float* h;               // [pairs x F]
    uint32_t* tops;         // [pairs x ceil(F/16)] largest magnitude of 16 features of H, fp32 bits
    uint8_t *xcodes, *hcodes;       // X and H quantized (where the products do not do it themselves), row-major, and their scales
    float *xscales, *hscales;
    uint16_t* Y;
};
constexpr int kFewUpStaged = 16 * 1024, kFewDownStaged = 64 * 1024;      // most codes that the products form and hold in LDS

// The experts that occur in the ids, in the order of their first occurrence: their number, and in list[i] the i-th
// one's id.  All threads of the workgroup take part; s_ids receives the ids, -1 for one out of range.
template <int THREADS>
__device__ __forceinline__ int distinct_experts(const W8FewArgs& a, int32_t* s_ids, int32_t* s_list, int32_t* s_count, bool* bad) {
    static_assert(THREADS >= kFewMaxPairs, "a thread per pair");
    const int tid = threadIdx.x, P = a.T * a.topk;
    int id = -1;
    if (tid < P) {
        id = a.ids[tid];
        if (id < 0 || id >= a.E) id = -1;
    }
    if (tid < kFewMaxPairs) s_ids[tid] = id;
    *bad = __syncthreads_or(tid < P && id < 0) != 0;
    bool first = id >= 0;
    if (tid < kFewMaxPairs)
        for (int q = 0; q < P; q += 4) {
            const int4 v = *reinterpret_cast<const int4*>(s_ids + q);       // (entries from P on are -1)
            first = first && !(v.x == id && q < tid) && !(v.y == id && q + 1 < tid) && !(v.z == id && q + 2 < tid) && !(v.w == id && q + 3 < tid);
        }
    const unsigned long long m = __builtin_amdgcn_ballot_w64(first);
    if ((tid & 63) == 0) s_count[tid >> 6] = __popcll(m);
    __syncthreads();
    int at = __popcll(m & ((1ull << (tid & 63)) - 1ull)), total = 0;
#pragma unroll
    for (int w = 0; w < kFewMaxPairs / 64; ++w) {
        at += w < (tid >> 6) ? s_count[w] : 0;
        total += s_count[w];
    }
    if (first) s_list[at] = id;
    __syncthreads();
    return total;
}
// The slot of token t that expert e is in (its first, if the caller repeats one), or -1.
__device__ __forceinline__ int slot_of(const int32_t* s_ids, int topk, int t, int e) {
    int found = -1;
    for (int j = topk - 1; j >= 0; --j) found = s_ids[t * topk + j] == e ? j : found;
    return found;
}

// Both kernels: column m of an operand of the matrix cores is token m.  Waves share the fragments of the weights in runs, 1 KB a
// fragment, and have the next run on its way.  No branch stands between the loads: what lies past an end is loaded from a
// clamped place and multiplied with zeros.  STAGED: the codes of the rows fit LDS, and the workgroup forms them there (so the
// layer takes two launches); else a launch of the row quantizer has formed them (every workgroup reads all of its rows, so the
// saving grows with the tokens).  Measured: 16 tokens to 8 experts of 14336 x 4096 read 940 MB in 164 us and 470 MB in 83 us, 5.7 TB/s;
// one token to 8 of 1408 x 2048 46 MB in 13.0 us and 23 MB in 11.9 us, where the trips to memory one after another (ids, table,
// activations, weights) count.
constexpr int kFewUpRun = 2, kFewDownRun = 4;

template <int IN, bool STAGED>
__global__ __launch_bounds__(kFewUpThreads, 4) void w8_few_up_kernel(const W8FewArgs a) {
    constexpr int NW = kFewUpThreads / 64, B = kFewUpRun;
    __shared__ __attribute__((aligned(16))) int32_t s_ids[kFewMaxPairs];
    __shared__ int32_t s_list[kFewMaxPairs], s_count[NW];
    __shared__ int32_t s_slot[kFewTokens];
    __shared__ uint32_t s_top[STAGED ? kFewTokens : 1][NW];
    __shared__ i32x4 s_part[2][NW][64];
    extern __shared__ __attribute__((aligned(16))) unsigned char codes[];   // piece c of 16 columns of token t: at (c * T + t) * 16
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int slot = blockIdx.y;
    bool bad;
    const int total = distinct_experts<kFewUpThreads>(a, s_ids, s_list, s_count, &bad);
    if (blockIdx.x == 0 && slot == 0 && tid == 0) a.status[0] = bad ? MILO_ERR_ROUTING : MILO_OK;
    if (slot >= total) return;
    const int e = __builtin_amdgcn_readfirstlane(s_list[slot]);
    const int kb = (int)w8_kblocks(a.H);
    const void* const p1 = a.experts[e].w1;
    const void* const p3 = a.experts[e].w3;
    if (tid < kFewTokens) s_slot[tid] = tid < a.T ? slot_of(s_ids, a.topk, tid, e) : -1;
    __syncthreads();
    const int m = lane & 15, c16 = lane >> 4;
    const bool mine = s_slot[m] >= 0;
    const int64_t wskip = (int64_t)blockIdx.x * kb * 1024;
    const GlobalFrag w1 = global_frag(reinterpret_cast<const char*>(p1) + wskip) + lane;
    const GlobalFrag w3 = global_frag(reinterpret_cast<const char*>(p3) + wskip) + lane;
    const BufRsrc rq = make_rsrc(a.xcodes, STAGED ? 0 : (uint64_t)a.T * kb * 64);
    u32x4 f1[2][B], f3[2][B], q[2][B];
    auto fetch = [&](int u, int to) {
#pragma unroll
        for (int i = 0; i < B; ++i) {
            const int v = u + i < kb ? u + i : kb - 1;
            f1[to][i] = w1[v * 64];
            f3[to][i] = w3[v * 64];
            if constexpr (!STAGED) {
                const uint32_t o = mine && u + i < kb ? (uint32_t)(m * kb * 64 + (u + i) * 64 + c16 * 16) : kOobOffset;
                q[to][i] = buf_load16(rq, o);
            }
        }
    };
    fetch(wave * B, 0);
    if constexpr (STAGED) {
        const char* const X = reinterpret_cast<const char*>(a.X);
        const int pieces = kb * 4;
        for (int t = 0; t < a.T; ++t) {
            if (s_slot[t] < 0) continue;
            uint32_t top = 0u;
            for (int p = tid; p < pieces; p += kFewUpThreads) top = raw_top<IN>(load16<IN>(X + t * a.H * 2, (int64_t)p * 16, a.H), top);
            top = wave_max(top_bits<IN>(top));
            if (lane == 0) s_top[t][wave] = top;
        }
        __syncthreads();
        for (int t = 0; t < a.T; ++t) {
            if (s_slot[t] < 0) continue;
            uint32_t top = s_top[t][0];
#pragma unroll
            for (int w = 1; w < NW; ++w) top = s_top[t][w] > top ? s_top[t][w] : top;
            const RowStep st = row_step(top);
            for (int p = tid; p < pieces; p += kFewUpThreads) {
                float v[16];
                raw_values<IN>(load16<IN>(X + t * a.H * 2, (int64_t)p * 16, a.H), v);
                *reinterpret_cast<u32x4*>(codes + (p * a.T + t) * 16) = row_codes16(v, st);
            }
        }
        __syncthreads();
    }
    float sx = 0.0f;
    if constexpr (STAGED) {
        if (mine) {
            uint32_t top = s_top[m][0];
#pragma unroll
            for (int w = 1; w < NW; ++w) top = s_top[m][w] > top ? s_top[m][w] : top;
            sx = row_step(top).s;
        }
    } else {
        if (mine) sx = a.xscales[m];
    }
    i32x4 acc1 = {0, 0, 0, 0}, acc3 = {0, 0, 0, 0};
    auto work = [&](int u, int from) {
        if constexpr (STAGED) {
#pragma unroll
            for (int i = 0; i < B; ++i) {
                q[from][i] = *reinterpret_cast<const u32x4*>(codes + (((u + i < kb ? u + i : 0) * 4 + c16) * a.T + (mine ? m : 0)) * 16);
                if (!mine || u + i >= kb) q[from][i] = u32x4{0u, 0u, 0u, 0u};
            }
        }
        fetch(u + B * NW, from ^ 1);
        asm volatile("" ::: "memory");              // (the loads stay in front)
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < B; ++i) {
            acc1 = mfma16_i8(f1[from][i], q[from][i], acc1);
            acc3 = mfma16_i8(f3[from][i], q[from][i], acc3);
        }
    };
    for (int u = wave * B; u < kb; u += 2 * B * NW) {
        work(u, 0);
        if (u + B * NW >= kb) break;
        work(u + B * NW, 1);
    }
    s_part[0][wave][lane] = acc1;
    s_part[1][wave][lane] = acc3;
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int i = 1; i < NW; ++i) {
        acc1 += s_part[0][i][lane];
        acc3 += s_part[1][i][lane];
    }
    const int64_t n = (int64_t)blockIdx.x * 16 + c16 * 4;
    uint32_t top = 0u;
    const int64_t row = mine ? m * a.topk + s_slot[m] : 0;
    if (mine) {
        const auto sw1 = global_float(w8_scales(p1, a.F, a.H) + n), sw3 = global_float(w8_scales(p3, a.F, a.H) + n);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (n + i >= a.F) continue;
            const float v = silu_times((float)acc1[i] * sx * sw1[i], (float)acc3[i] * sx * sw3[i]);
            a.h[row * a.F + n + i] = v;
            const uint32_t b = __float_as_uint(v) & 0x7fffffffu;
            top = b > top ? b : top;
        }
    }
#pragma unroll
    for (int d = 16; d <= 32; d <<= 1) {
        const uint32_t o = __shfl_xor(top, d, 64);
        top = o > top ? o : top;
    }
    if (mine && c16 == 0) a.tops[row * ((a.F + 15) / 16) + blockIdx.x] = top;
}

// The runs of all experts' weights are one sequence, which the waves share.  The products of a run are added up in integers; what one expert's runs
// add up to, and the experts, in 64 bits: a linear's sum is to be that of the integers, and its pieces may cancel.
template <bool BF, bool STAGED>
__global__ __launch_bounds__(kFewDownThreads, 4) void w8_few_down_kernel(const W8FewArgs a) {
    constexpr int NW = kFewDownThreads / 64, B = kFewDownRun;
    __shared__ __attribute__((aligned(16))) int32_t s_ids[kFewMaxPairs];
    __shared__ int32_t s_list[kFewMaxPairs], s_count[NW];
    __shared__ RowStep s_step[STAGED ? kFewMaxPairs : 1];           // per pair
    __shared__ uint64_t s_w[kFewMaxPairs];                          // per expert that occurs: its weight,
    __shared__ __attribute__((aligned(16))) float s_sw[kFewMaxPairs][16];   // the scales of this workgroup's features,
    __shared__ int32_t s_row[kFewMaxPairs][kFewTokens];             // its tokens' rows (-1: none)
    __shared__ float s_factor[kFewMaxPairs][kFewTokens];            // and the rows' scales times the gates
    __shared__ f64x4 s_part[NW][64];
    extern __shared__ __attribute__((aligned(16))) unsigned char codes[];   // piece c of 16 columns of pair p: at (c * P + p) * 16
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int kb = (int)w8_kblocks(a.F), P = a.T * a.topk;
    if constexpr (STAGED) {
        const int nt = (int)((a.F + 15) / 16);
        for (int p = wave; p < P; p += NW) {        // (a pair that has no row: some value, which nothing uses)
            uint32_t top = 0u;
            const uint32_t* const tops = a.tops + (int64_t)p * nt;
            for (int i = lane; i < nt; i += 64) top = tops[i] > top ? tops[i] : top;
            top = wave_max(top);
            if (lane == 0) s_step[p] = row_step(top);
        }
    }
    bool bad;
    const int total = distinct_experts<kFewDownThreads>(a, s_ids, s_list, s_count, &bad);
    for (int i = tid; i < total * 16; i += kFewDownThreads) {
        const int s = i >> 4, m = i & 15, e = s_list[s];
        const void* const w = a.experts[e].w2;
        if (m == 0) s_w[s] = (uint64_t)(uintptr_t)w;
        s_sw[s][m] = global_float(w8_scales(w, a.H, a.F))[(int64_t)blockIdx.x * 16 + m];
        const int j = m < a.T ? slot_of(s_ids, a.topk, m, e) : -1, row = j >= 0 ? m * a.topk + j : -1;
        float f = 0.0f;
        if (j >= 0) {
            for (int k = j; k < a.topk; ++k) f += s_ids[m * a.topk + k] == e ? a.gates[m * a.topk + k] : 0.0f;
            f *= STAGED ? s_step[row].s : a.hscales[row];
        }
        s_row[s][m] = row;
        s_factor[s][m] = f;
    }
    __syncthreads();
    // run r: fragments B (r % runs) .. of expert r / runs
    const int m = lane & 15, c16 = lane >> 4;
    const int runs = (kb + B - 1) / B, all = total * runs;
    const int64_t skip = (int64_t)blockIdx.x * kb * 64 + lane;
    const BufRsrc rq = make_rsrc(a.hcodes, STAGED ? 0 : (uint64_t)P * kb * 64);
    u32x4 w[2][B], q[2][B];
    auto fetch = [&](int r, int to) {
        r = r < all ? r : all - 1;
        const int s = r / runs, u = (r - s * runs) * B;
        const GlobalFrag p = global_frag((const void*)(uintptr_t)s_w[s]) + skip;
#pragma unroll
        for (int i = 0; i < B; ++i) w[to][i] = p[(u + i < kb ? u + i : kb - 1) * 64];
        if constexpr (!STAGED) {
            const int row = s_row[s][m];
#pragma unroll
            for (int i = 0; i < B; ++i) {
                const uint32_t o = row >= 0 && u + i < kb ? (uint32_t)row * (uint32_t)(kb * 64) + (uint32_t)((u + i) * 64 + c16 * 16) : kOobOffset;
                q[to][i] = buf_load16(rq, o);
            }
        }
    };
    if (all > 0) fetch(wave, 0);
    if constexpr (STAGED) {
        // four values a thread: neighbours are the quarters of a piece, then the pairs
        const int n = P * kb * 16;
#pragma unroll 4
        for (int i = tid; i < n; i += kFewDownThreads) {
            const int c = (i >> 2) / P, p = (i >> 2) - c * P;
            const int64_t k = (int64_t)c * 16 + (i & 3) * 4;
            const float* const h = a.h + (int64_t)p * a.F + k;
            float v[4];
            if (k + 4 <= a.F) {
                __builtin_memcpy(v, h, 16);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j) v[j] = k + j < a.F ? h[j] : 0.0f;
            }
            *reinterpret_cast<uint32_t*>(codes + i * 4) = row_codes4(v, s_step[p]);
        }
        __syncthreads();
    }
    f64x4 y = {0.0, 0.0, 0.0, 0.0};
    auto work = [&](int r, int from) {
        const int s = r / runs, u = (r - s * runs) * B;
        const float f = s_factor[s][m];
        const int row = s_row[s][m];
        const f32x4 sw = *reinterpret_cast<const f32x4*>(&s_sw[s][c16 * 4]);
        if constexpr (STAGED) {
#pragma unroll
            for (int i = 0; i < B; ++i) {
                q[from][i] = *reinterpret_cast<const u32x4*>(codes + (((u + i < kb ? u + i : 0) * 4 + c16) * P + (row >= 0 ? row : 0)) * 16);
                if (row < 0 || u + i >= kb) q[from][i] = u32x4{0u, 0u, 0u, 0u};
            }
        }
        fetch(r + NW, from ^ 1);
        asm volatile("" ::: "memory");              // (the loads stay in front)
        __builtin_amdgcn_sched_barrier(0);
        i32x4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int i = 0; i < B; ++i) acc = mfma16_i8(w[from][i], q[from][i], acc);
#pragma unroll
        for (int i = 0; i < 4; ++i) y[i] += row >= 0 ? (double)acc[i] * ((double)f * (double)sw[i]) : 0.0;      // (another token's expert may have a scale that is no number)
    };
    for (int r = wave; r < all; r += 2 * NW) {
        work(r, 0);
        if (r + NW >= all) break;
        work(r + NW, 1);
    }
    s_part[wave][lane] = y;
    __syncthreads();
    const int64_t n = (int64_t)blockIdx.x * 16 + c16 * 4;
    if (wave != 0 || m >= a.T || n >= a.H) return;
#pragma unroll
    for (int i = 1; i < NW; ++i) y += s_part[i][lane];
    const float v[4] = {(float)y[0], (float)y[1], (float)y[2], (float)y[3]};
    store4<BF>(a.Y + m * a.H + n, v, (int)(a.H - n < 4 ? a.H - n : 4), (a.H & 3) == 0);
}
template <bool BF, bool STAGED>
static int launch_few_down(const W8FewArgs& a, dim3 grid, int lds, hipStream_t stream) {
    if constexpr (STAGED) {
        static bool raised[64] = {false};
        const int st = raise_lds(reinterpret_cast<const void*>(w8_few_down_kernel<BF, STAGED>), kFewDownStaged, raised);
        if (st != MILO_OK) return st;
    }
    w8_few_down_kernel<BF, STAGED><<<grid, dim3(kFewDownThreads), lds, stream>>>(a);
    return launch_status();
}
template <int IN>
static int launch_few(const W8FewArgs& a, hipStream_t s) {
    const int P = a.T * a.topk;
    const dim3 gu((unsigned)((a.F + 15) / 16), (unsigned)(P < a.E ? P : a.E)), gd((unsigned)((a.H + 15) / 16));
    W8QuantArgs q;
    q.blocked = 0;
    const int xbytes = a.T * (int)w8_kblocks(a.H) * 64;
    if (xbytes <= kFewUpStaged) {
        w8_few_up_kernel<IN, true><<<gu, dim3(kFewUpThreads), xbytes, s>>>(a);
    } else {
        q.in = a.X;
        q.rows = a.T;
        q.K = a.H;
        q.codes = a.xcodes;
        q.scales = a.xscales;
        const int st = launch_w8_quant(q, IN, s);
        if (st != MILO_OK) return st;
        w8_few_up_kernel<IN, false><<<gu, dim3(kFewUpThreads), 0, s>>>(a);
    }
    int st = launch_status();
    if (st != MILO_OK) return st;
    const int bytes = P * (int)w8_kblocks(a.F) * 64;
    if (bytes <= kFewDownStaged) return launch_few_down<IN == W8_BF16, true>(a, gd, bytes, s);
    q.in = a.h;
    q.rows = P;
    q.K = a.F;
    q.codes = a.hcodes;
    q.scales = a.hscales;
    st = launch_w8_quant(q, W8_F32, s);
    if (st != MILO_OK) return st;
    return launch_few_down<IN == W8_BF16, false>(a, gd, 0, s);
}

// ---------------------------------------------------------------------------------------------
// Y = sum over a token's pairs of their rows of O, in slot order; a pair whose id is out of range has none.
template <bool BF>
__global__ __launch_bounds__(256) void w8_combine_kernel(const float* __restrict__ O, const int32_t* __restrict__ ids, int topk, int E, int64_t H,
                                                         uint16_t* __restrict__ Y) {
    const int64_t t = blockIdx.x;
    for (int64_t h = (int64_t)threadIdx.x * 4; h < H; h += 1024) {
        const int left = (int)(H - h < 4 ? H - h : 4);
        float v[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (int j = 0; j < topk; ++j) {
            const int64_t p = t * topk + j;
            if ((uint32_t)ids[p] >= (uint32_t)E) continue;
            const float* const o = O + p * H + h;
            float r[4] = {0.0f, 0.0f, 0.0f, 0.0f};
            if (left == 4) {
                __builtin_memcpy(r, o, 16);
            } else {
#pragma unroll
                for (int i = 0; i < 4; ++i)
                    if (i < left) r[i] = o[i];
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) v[i] += r[i];
        }
        store4<BF>(Y + t * H + h, v, left, (H & 3) == 0);
    }
}

// Order of the grouped products' tiles.  A third to a half of the slots are empty, and with most experts at one tile every second one is: with the
// rows fastest the workgroups that do work then land on every second place that the dispatcher deals out, which it does in turn,
// and half of the compute units idle.  Runs of eight columns keep an XCD's places even and its tiles of one expert close enough to share the weight; groups
// of many slots spread every expert over all XCDs.  8 experts of 14336 x 4096: gate and up at 128 rows each 281 us with the rows
// fastest in groups of 8, 203 so; the layer at 512 tokens 457 and 419, with 128 rows each 457 and 377, at 64 tokens 327 and 265; 4096 tokens
// of 66 x 1408 x 2048 585 and 546.
constexpr int kGroupM = 64, kSpan = 8;

// Workspace of a forward.
struct W8MoeLayout {
    bool few;
    W8Kernel kernel;
    int bm, max_tiles;
    size_t off_status, off_tops, off_h, off_xq, off_xs, off_sorted, off_token, off_tiles, off_hq, off_hs, off_o, total;
};
static bool w8_moe_layout(int64_t T, int64_t H, int64_t F, int E, int topk, W8MoeLayout* L) {
    if (T < 1 || E < 1 || E > 65536 || topk < 1 || topk > E) return false;
    if (!w8_shape_ok(F, H) || !w8_shape_ok(H, F)) return false;
    if (T >= (int64_t(1) << 23) || T > (int64_t(1) << 30) / topk) return false;
    if (E > (int64_t(1) << 27) / (H > F ? H : F)) return false;
    const int64_t P = T * topk, hb = w8_kblocks(H) * 64, fb = w8_kblocks(F) * 64;
    // rows of codes are addressed with 32-bit offsets
    if (T * hb >= 0xFFFF0000ll || P * fb >= 0xFFFF0000ll) return false;
    size_t off = 256;
    L->off_status = 0;
    auto take = [&](size_t bytes) {
        const size_t at = off;
        off = align_up(off + bytes, 256);
        return at;
    };
    L->few = T <= kFewTokens && P <= kFewMaxPairs;
    // Rows per expert decide, on average, as the host knows no other number: the weights' bytes bound a few of them, and tiles of 32 x 64 have them on
    // their way soonest.  In those and in tiles of 128 x 256, us, ids of equal popularity / popularity falling with the rank (the most popular expert has
    // three to eight times the mean):
    //   8 experts of 14336 x 4096    12 rows 257 and 290 / 263 and 287    20: 272 and 297 / 292 and 309    32: 323 and 305 / 333 and 332
    //   66 of 1408 x 2048, 2 shared  12 rows 139 and 143 / 112 and 112    20: 150 and 149 / 132 and 127    32: 166 and 155 / 160 and 139
    //   32 of 4096 x 1024            12 rows 108 and 108 /  95 and  99    20: 114 and 110 / 111 and 111    32: 135 and 114 / 142 and 122
    //   17 of 2730 x 1000, 1 shared  12 rows  49 and  49 /  49 and  50    20:  52 and  55 /  53 and  55    32:  57 and  59 /  60 and  60
    // Just below 24 rows the small tiles cost up to 11 % more than the large ones (24 rows of 66 experts: 157 and 151 / 144 and 130), just above it the large ones up to
    // 5 % (8 experts: 285 and 300 / 304 and 318).
    L->kernel = P < 24 * (P < E ? P : E) ? W8_WIDE_32x64 : W8_TILE_128x256;
    // The grid has workgroups for every slot of the list of tiles, some of them empty.  Where those of the small tiles are too many (thousands of
    // experts of long rows), the large ones, which are a quarter as many, serve; where those are, the call is refused before it launches anything.
    auto tile_rows = [](W8Kernel k) { return k == W8_WIDE_32x64 ? 32 : 128; };
    auto fits = [&](W8Kernel k) {       // gate and up (half as many features of either), down
        const int64_t slots = (P + tile_rows(k) - 1) / tile_rows(k) + E, down = k == W8_WIDE_32x64 ? 64 : 256, up = down / 2;
        return slots * ((F + up - 1) / up) <= kW8MaxGroups && slots * ((H + down - 1) / down) <= kW8MaxGroups;
    };
    if (!L->few && !fits(L->kernel)) L->kernel = W8_TILE_128x256;
    if (!L->few && !fits(L->kernel)) return false;
    L->off_h = take((size_t)P * F * 4);
    L->off_xq = take((size_t)(T * hb));
    L->off_xs = take((size_t)T * 4);
    if (L->few) {
        L->off_tops = take((size_t)P * ((F + 15) / 16) * 4);
        L->off_hq = take((size_t)(P * fb));
        L->off_hs = take((size_t)P * 4);
    } else {
        L->bm = tile_rows(L->kernel);
        L->max_tiles = (int)((P + L->bm - 1) / L->bm) + E;
        L->off_sorted = take((size_t)P * 4);
        L->off_token = take((size_t)P * 4);
        L->off_tiles = take((size_t)L->max_tiles * sizeof(TileDesc));
        L->off_hq = take((size_t)(P * fb));
        L->off_hs = take((size_t)P * 4);
        L->off_o = take((size_t)P * H * 4);
    }
    L->total = off;
    return true;
}

}  // namespace milo

using namespace milo;

extern "C" int milo_moe_w8a8_check_experts(const milo_w8_expert* experts, int E, int64_t H, int64_t F) {
    if (!experts) return MILO_ERR_NULL;
    if (E < 1 || E > 65536 || !w8_shape_ok(F, H) || !w8_shape_ok(H, F)) return MILO_ERR_SHAPE;
    for (int e = 0; e < E; ++e) {
        if (!experts[e].w1 || !experts[e].w3 || !experts[e].w2) return MILO_ERR_NULL;
        if (!aligned16(experts[e].w1) || !aligned16(experts[e].w3) || !aligned16(experts[e].w2)) return MILO_ERR_ALIGN;
    }
    return MILO_OK;
}

extern "C" size_t milo_moe_w8a8_workspace(int64_t T, int64_t H, int64_t F, int E, int topk) {
    W8MoeLayout L;
    return w8_moe_layout(T, H, F, E, topk, &L) ? L.total : 0;
}

extern "C" int milo_moe_w8a8_forward(const milo_half* X, int64_t T, int64_t H, int64_t F, const milo_w8_expert* experts, int E, const int32_t* topk_ids,
                                     const float* topk_weights, int topk, unsigned flags, milo_half* Y, int32_t* status, void* workspace, size_t workspace_bytes,
                                     void* stream) {
    if (!X || !experts || !topk_ids || !topk_weights || !Y) return MILO_ERR_NULL;
    W8MoeLayout L;
    if ((flags & ~MILO_ACT_BF16) || !w8_moe_layout(T, H, F, E, topk, &L)) return MILO_ERR_SHAPE;
    if (!workspace || workspace_bytes < L.total) return MILO_ERR_WORKSPACE;
    if (!aligned16(X) || !aligned16(experts) || !aligned16(topk_ids) || !aligned16(topk_weights) || !aligned16(Y) || !aligned16(status) || !aligned16(workspace)) return MILO_ERR_ALIGN;
    const bool bf = (flags & MILO_ACT_BF16) != 0;
    const hipStream_t s = (hipStream_t)stream;
    char* const ws = reinterpret_cast<char*>(workspace);
    if (!status) status = reinterpret_cast<int32_t*>(ws + L.off_status);
    const int64_t P = T * topk;
    if (L.few) {
        W8FewArgs a;
        a.X = X;
        a.T = (int)T;
        a.topk = topk;
        a.E = E;
        a.H = H;
        a.F = F;
        a.experts = experts;
        a.ids = topk_ids;
        a.gates = topk_weights;
        a.status = status;
        a.h = reinterpret_cast<float*>(ws + L.off_h);
        a.tops = reinterpret_cast<uint32_t*>(ws + L.off_tops);
        a.xcodes = reinterpret_cast<uint8_t*>(ws + L.off_xq);
        a.xscales = reinterpret_cast<float*>(ws + L.off_xs);
        a.hcodes = reinterpret_cast<uint8_t*>(ws + L.off_hq);
        a.hscales = reinterpret_cast<float*>(ws + L.off_hs);
        a.Y = Y;
        return bf ? launch_few<W8_BF16>(a, s) : launch_few<W8_F16>(a, s);
    }
    W8QuantArgs q;
    q.in = X;
    q.rows = T;
    q.K = H;
    q.codes = reinterpret_cast<uint8_t*>(ws + L.off_xq);
    q.scales = reinterpret_cast<float*>(ws + L.off_xs);
    q.blocked = 0;
    int st = launch_w8_quant(q, bf ? W8_BF16 : W8_F16, s);
    if (st != MILO_OK) return st;
    RouteArgs g = {};
    g.ids = topk_ids;
    g.P = (int32_t)P;
    g.E = E;
    g.bm = L.bm;
    g.topk = topk;
    g.sorted = reinterpret_cast<int32_t*>(ws + L.off_sorted);
    g.sorted_token = reinterpret_cast<int32_t*>(ws + L.off_token);
    g.tiles = reinterpret_cast<TileDesc*>(ws + L.off_tiles);
    g.header = status;
    g.max_tiles = L.max_tiles;
    st = launch_pair_groups(g, s);
    if (st != MILO_OK) return st;
    W8TileArgs t = {};
    t.A = q.codes;
    t.a_bytes = (uint64_t)(T * w8_kblocks(H) * 64);
    t.a_scales = q.scales;
    t.N = F;
    t.K = H;
    t.experts = experts;
    t.tiles = g.tiles;
    t.m_tiles = L.max_tiles;
    t.group_m = kGroupM;
    t.span = kSpan;
    t.x_rows = g.sorted_token;
    t.out = ws + L.off_h;
    st = launch_w8_product(t, 1, L.kernel, s);
    if (st != MILO_OK) return st;
    q.in = ws + L.off_h;
    q.rows = P;
    q.K = F;
    q.codes = reinterpret_cast<uint8_t*>(ws + L.off_hq);
    q.scales = reinterpret_cast<float*>(ws + L.off_hs);
    st = launch_w8_quant(q, W8_F32, s);
    if (st != MILO_OK) return st;
    t.A = q.codes;
    t.a_bytes = (uint64_t)(P * w8_kblocks(F) * 64);
    t.a_scales = q.scales;
    t.N = H;
    t.K = F;
    t.x_rows = g.sorted;
    t.gates = topk_weights;
    t.out = ws + L.off_o;
    st = launch_w8_product(t, 2, L.kernel, s);
    if (st != MILO_OK) return st;
    auto combine = [&](auto kernel) { kernel<<<dim3((unsigned)T), dim3(256), 0, s>>>(reinterpret_cast<const float*>(ws + L.off_o), topk_ids, topk, E, H, Y); };
    if (bf) combine(w8_combine_kernel<true>);
    else combine(w8_combine_kernel<false>);
    return launch_status();
}

// For the tests: the kernel of a layer's grouped products (W8Kernel), -1 for those of a few tokens, -2 for a shape that is refused.
extern "C" int milo_moe_w8a8_route(int64_t T, int64_t H, int64_t F, int E, int topk) {
    W8MoeLayout L;
    if (!w8_moe_layout(T, H, F, E, topk, &L)) return -2;
    return L.few ? -1 : (int)L.kernel;
}
