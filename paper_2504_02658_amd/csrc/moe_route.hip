// milo_moe_route: which experts a token goes to, and with what weight.
//
//   l[t][e] = sum_k X[t][k] Wg[e][k],  ids = the topk largest l (equal ones: the lowest id first),
//   gates = exp(l_chosen - max l) / sum over all experts (or over the chosen ones) of exp(l - max l)
//
// Whether two logits are in one order or the other decides which weights a token meets, so the sums are held in 64 bits:
// products of two 16-bit numbers are exact there, and so are the sums while they fit 53 bits.  (The kernels below add in different orders: beyond
// that, logits that differ by 64-bit rounding may change places between them.)
#include "milo_host.h"
#include "w8_kernels.h"

namespace milo {

constexpr int kRouteMaxExperts = 1024, kRouteMaxTopk = 64;
constexpr int kGateThreads = 1024;

struct GateArgs {
    const void* X;
    const void* Wg;
    int64_t T, H;
    int E, topk, n_shared, renormalize;
    int32_t* ids;
    float* gates;
};

// Order of logits as signed integers: NaN below everything, the two zeros equal.
__device__ __forceinline__ int64_t logit_key(double l) {
    const int64_t b = __builtin_bit_cast(int64_t, l + 0.0);
    if (l != l) return INT64_MIN;
    return b < 0 ? (b ^ INT64_MAX) : b;
}

// Largest value of a wave, by rows of 16 and then across them, in every lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t max_step(int64_t v) {
    const int lo = (int)(uint32_t)v, hi = (int)(v >> 32);
    const uint32_t olo = (uint32_t)__builtin_amdgcn_update_dpp(lo, lo, CTRL, ROWS, 0xf, false);
    const int ohi = __builtin_amdgcn_update_dpp(hi, hi, CTRL, ROWS, 0xf, false);
    const int64_t o = (int64_t)ohi << 32 | olo;
    return o > v ? o : v;
}
__device__ __forceinline__ int64_t wave_max_key(int64_t v) {
    v = max_step<0x111, 0xf>(v);        // row_shr 1, 2, 4, 8: lane 15 of a row has the row's
    v = max_step<0x112, 0xf>(v);
    v = max_step<0x114, 0xf>(v);
    v = max_step<0x118, 0xf>(v);
    v = max_step<0x142, 0xa>(v);        // row_bcast 15 and 31: lane 63 has the wave's
    v = max_step<0x143, 0xc>(v);
    const uint32_t lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, 63);
    const int hi = __builtin_amdgcn_readlane((int)(v >> 32), 63);
    return (int64_t)hi << 32 | lo;
}

// One wave chooses from logits[0, E) of one token and writes the token's row of ids and gates.
__device__ __forceinline__ void choose_experts(const double* logits, int64_t t, const GateArgs& a) {
    const int lane = threadIdx.x & 63, width = a.topk + a.n_shared;
    uint32_t taken = 0u;        // of expert lane + 64 i: bit i
    int my_id = 0;
    double top = 0.0, my_logit = 0.0;
    int64_t key = INT64_MIN;    // of this lane's best expert that is left, and the expert (-1: none)
    int id = -1;
    auto best_left = [&] {
        key = INT64_MIN;
        id = -1;
        for (int i = 0, e = lane; e < a.E; ++i, e += 64)
            if (!(taken >> i & 1)) {
                const int64_t k = logit_key(logits[e]);
                if (k > key || id < 0) {
                    key = k;
                    id = e;
                }
            }
    };
    best_left();
    for (int j = 0; j < a.topk; ++j) {
        const int64_t most = wave_max_key(key);
        // (topk <= E: some lane has it; of equal ones the lowest id)
        unsigned long long m = __builtin_amdgcn_ballot_w64(id >= 0 && key == most);
        int first = 0x7fffffff;
        while (m) {
            const int e = __builtin_amdgcn_readlane(id, (int)__builtin_ctzll(m));
            first = e < first ? e : first;
            m &= m - 1;
        }
        const double l = logits[first];
        if (j == 0) top = l;
        if (lane == j) {
            my_id = first;
            my_logit = l;
        }
        if ((first & 63) == lane) {
            taken |= 1u << (first >> 6);
            best_left();
        }
    }
    // (a NaN logit, infinite ones or a NaN in the inputs: every gate of the token is NaN, as the quotient gives)
    double sum = 0.0;
    bool nan = false;
    // exp in 64 bits: rounded to fp32, the argument of an expert far from the top would move its gate by the distance's own rounding.
    const double mine = lane < a.topk ? exp(my_logit - top) : 0.0;
    for (int e = lane; e < a.E; e += 64) {
        const double l = logits[e];
        nan = nan || l != l;
        if (!a.renormalize) sum += exp(l - top);
    }
    if (a.renormalize) sum = mine;
    if (nan) sum = __builtin_nan("");
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) sum += __shfl_xor(sum, d, 64);
    if (lane < a.topk) {
        a.ids[t * width + lane] = my_id;
        a.gates[t * width + lane] = (float)(mine / sum);
    }
    for (int j = lane; j < a.n_shared; j += 64) {
        a.ids[t * width + a.topk + j] = a.E + j;
        a.gates[t * width + a.topk + j] = 1.0f;
    }
}

// Eight elements [k, k + 8) of a row of H, zeros beyond it.
__device__ __forceinline__ u32x4 load8(const char* row, int64_t k, int64_t H) {
    u32x4 r = {0u, 0u, 0u, 0u};
    if (k + 8 <= H) {
        __builtin_memcpy(&r, row + k * 2, 16);
    } else {
        const uint16_t* const p = reinterpret_cast<const uint16_t*>(row);
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (k + i < H) r[i >> 1] |= (uint32_t)p[k + i] << (16 * (i & 1));
    }
    return r;
}
template <int IN>
__device__ __forceinline__ double value8(const u32x4& r, int i) {
    if constexpr (IN == W8_F16) return (double)(float)f16_bits((r[i >> 1] >> (16 * (i & 1))) & 0xffffu);
    else return (double)__uint_as_float(i & 1 ? r[i >> 1] & 0xffff0000u : r[i >> 1] << 16);
}

// Few tokens: a workgroup per token, whose waves take four experts at a time, lanes along H.  Latency, and one compute unit's read of
// the router's weight, bound it.
template <int IN>
__global__ __launch_bounds__(kGateThreads) void moe_gate_token_kernel(const GateArgs a) {
    constexpr int G = 4;
    __shared__ double s_logit[kRouteMaxExperts];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = blockIdx.x;
    const char* const x = reinterpret_cast<const char*>(a.X) + t * a.H * 2;
    for (int e0 = wave * G; e0 < a.E; e0 += kGateThreads / 64 * G) {
        const char* w[G];
#pragma unroll
        for (int g = 0; g < G; ++g) w[g] = reinterpret_cast<const char*>(a.Wg) + (int64_t)(e0 + g < a.E ? e0 + g : a.E - 1) * a.H * 2;
        double l[G] = {0.0, 0.0, 0.0, 0.0};
#pragma unroll 2
        for (int64_t k = lane * 8; k < a.H; k += 512) {
            const u32x4 xr = load8(x, k, a.H);
            u32x4 wr[G];
#pragma unroll
            for (int g = 0; g < G; ++g) wr[g] = load8(w[g], k, a.H);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const double v = value8<IN>(xr, i);
#pragma unroll
                for (int g = 0; g < G; ++g) l[g] = fma(v, value8<IN>(wr[g], i), l[g]);
            }
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1)
#pragma unroll
            for (int g = 0; g < G; ++g) l[g] += __shfl_xor(l[g], d, 64);
#pragma unroll
        for (int g = 0; g < G; ++g)
            if (lane == 0 && e0 + g < a.E) s_logit[e0 + g] = l[g];
    }
    __syncthreads();
    if (wave == 0) choose_experts(s_logit, t, a);
}

// Many tokens: a workgroup takes 16 of them to all experts on the 64-bit matrix instructions, 16 TILES experts at a time; its waves share H in
// blocks of 32, of which lane (row, q) holds elements 8q .. 8q + 7 of its row, so that step j multiplies element j of every quarter.
// The rate of those instructions bounds it (64 multiplications per cycle and compute unit).
constexpr int kGateTileWaves = 8, kGateTileExperts = 256;
template <int IN, int TILES>
__global__ __launch_bounds__(kGateTileWaves * 64) void moe_gate_tile_kernel(const GateArgs a) {
    __shared__ double s_logit[16][kGateTileExperts];
    extern __shared__ __attribute__((aligned(32))) unsigned char smem[];
    f64x4* const s_part = reinterpret_cast<f64x4*>(smem);           // [wave][tile][lane]
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int r16 = lane & 15, q = lane >> 4;
    const int64_t t0 = (int64_t)blockIdx.x * 16;
    const int64_t row = t0 + r16 < a.T ? t0 + r16 : a.T - 1;
    const char* const x = reinterpret_cast<const char*>(a.X) + row * a.H * 2;
    for (int e0 = 0; e0 < a.E; e0 += 16 * TILES) {
        const char* w[TILES];
#pragma unroll
        for (int i = 0; i < TILES; ++i) {
            const int e = e0 + 16 * i + r16;
            w[i] = reinterpret_cast<const char*>(a.Wg) + (int64_t)(e < a.E ? e : a.E - 1) * a.H * 2;
        }
        f64x4 acc[TILES];
#pragma unroll
        for (int i = 0; i < TILES; ++i) acc[i] = f64x4{0.0, 0.0, 0.0, 0.0};
        u32x4 xr[2], wr[2][TILES];
        auto fetch = [&](int64_t k, int to) {
            xr[to] = load8(x, k + q * 8, a.H);
#pragma unroll
            for (int i = 0; i < TILES; ++i) wr[to][i] = load8(w[i], k + q * 8, a.H);
        };
        auto work = [&](int64_t k, int from) {
            fetch(k + kGateTileWaves * 32, from ^ 1);
            asm volatile("" ::: "memory");              // (the loads stay in front)
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const double v = value8<IN>(xr[from], j);
#pragma unroll
                for (int i = 0; i < TILES; ++i) acc[i] = __builtin_amdgcn_mfma_f64_16x16x4f64(value8<IN>(wr[from][i], j), v, acc[i], 0, 0, 0);
                __builtin_amdgcn_sched_barrier(0);
            }
        };
        fetch(wave * 32, 0);
        for (int64_t k = wave * 32; k < a.H; k += 2 * kGateTileWaves * 32) {
            work(k, 0);
            if (k + kGateTileWaves * 32 >= a.H) break;
            work(k + kGateTileWaves * 32, 1);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < TILES; ++i) s_part[(wave * TILES + i) * 64 + lane] = acc[i];
        __syncthreads();
        // lane (token r16, q) of tile i: experts 16 i + 4 j + q
        for (int i = wave; i < TILES; i += kGateTileWaves) {
            f64x4 s = s_part[i * 64 + lane];
#pragma unroll
            for (int v = 1; v < kGateTileWaves; ++v) s += s_part[(v * TILES + i) * 64 + lane];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int e = e0 + 16 * i + 4 * j + q;
                if (e < a.E) s_logit[r16][e] = s[j];
            }
        }
    }
    __syncthreads();
    for (int t = wave; t < 16; t += kGateTileWaves)
        if (t0 + t < a.T) choose_experts(s_logit[t], t0 + t, a);
}

template <int IN, int TILES>
static int launch_gate_tile(const GateArgs& a, hipStream_t stream) {
    constexpr int lds = kGateTileWaves * TILES * 64 * sizeof(f64x4);
    static bool raised[64] = {false};
    const int st = raise_lds(reinterpret_cast<const void*>(moe_gate_tile_kernel<IN, TILES>), lds, raised);
    if (st != MILO_OK) return st;
    moe_gate_tile_kernel<IN, TILES><<<dim3((unsigned)((a.T + 15) / 16)), dim3(kGateTileWaves * 64), lds, stream>>>(a);
    return launch_status();
}
template <int IN>
static int launch_gate(const GateArgs& a, hipStream_t stream) {
    // A workgroup per token reads the weight once per token, 16 tokens share it.  Both sides, us, at 512, 1024 and 4096 tokens: 64 experts of 2048 18, 31, 108
    // and 30, 30, 31; 8 of 4096 12, 21, 77 and 18, 18, 20; 64 of 512 11, 18, 56 and 16; 128 of 4096 54, 99, 340 and 93; 256 of 7168 160, 301, 1099 and
    // 290: they meet between 750 and 1050 tokens.  More than 256 experts have no room for their logits beside each other: 512 of 2048, 4096
    // tokens, 769.
    if (a.T > 1024 && a.E <= kGateTileExperts) return a.E <= 16 ? launch_gate_tile<IN, 1>(a, stream) : launch_gate_tile<IN, 4>(a, stream);
    moe_gate_token_kernel<IN><<<dim3((unsigned)a.T), dim3(kGateThreads), 0, stream>>>(a);
    return launch_status();
}

}  // namespace milo

using namespace milo;

extern "C" int milo_moe_route(const milo_half* X, int64_t T, int64_t H, const milo_half* Wg, int E, int topk, int n_shared, unsigned flags,
                              int32_t* ids, float* gates, void* stream) {
    if (!X || !Wg || !ids || !gates) return MILO_ERR_NULL;
    if (T < 1 || T >= (int64_t(1) << 22) || H < 1 || H > (int64_t(1) << 20) || E < 1 || E > kRouteMaxExperts || topk < 1 || topk > E || topk > kRouteMaxTopk ||
        n_shared < 0 || n_shared > kRouteMaxTopk || (flags & ~(MILO_ACT_BF16 | MILO_ROUTE_RENORMALIZE)))
        return MILO_ERR_SHAPE;
    if (!aligned16(X) || !aligned16(Wg) || !aligned16(ids) || !aligned16(gates)) return MILO_ERR_ALIGN;
    GateArgs a;
    a.X = X;
    a.Wg = Wg;
    a.T = T;
    a.H = H;
    a.E = E;
    a.topk = topk;
    a.n_shared = n_shared;
    a.renormalize = (flags & MILO_ROUTE_RENORMALIZE) != 0;
    a.ids = ids;
    a.gates = gates;
    return flags & MILO_ACT_BF16 ? launch_gate<W8_BF16>(a, (hipStream_t)stream) : launch_gate<W8_F16>(a, (hipStream_t)stream);
}
