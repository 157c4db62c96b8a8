// milo_moe_route: which experts a token goes to, and with what weight.
//
//   l[t][e] = sum_k X[t][k] Wg[e][k],  ids = the topk largest l (equal ones: the lowest id first),
//   gates = exp(l_chosen - max l) / sum over all experts (or over the chosen ones) of exp(l - max l)
//
// Whether two logits are in one order or the other decides which weights a token meets, so the sums are held in 64 bits:
// products of two 16-bit numbers are exact there, and the choice does not hang on the order of the summation.
#include "milo_host.h"
#include "w8_kernels.h"

namespace milo {

constexpr int kRouteMaxExperts = 1024, kRouteMaxTopk = 64;
constexpr int kGateThreads = 256;

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

// One wave chooses from logits[0, E) of one token and writes the token's row of ids and gates.
__device__ __forceinline__ void choose_experts(const double* logits, int64_t t, const GateArgs& a) {
    const int lane = threadIdx.x & 63, width = a.topk + a.n_shared;
    uint32_t taken = 0u;        // of expert lane + 64 i: bit i
    int my_id = 0;
    double top = 0.0, my_logit = 0.0;
    for (int j = 0; j < a.topk; ++j) {
        int64_t key = INT64_MIN;
        int id = 0x7fffffff;
        for (int i = 0, e = lane; e < a.E; ++i, e += 64)
            if (!(taken >> i & 1)) {
                const int64_t k = logit_key(logits[e]);
                if (k > key || id == 0x7fffffff) {
                    key = k;
                    id = e;
                }
            }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) {
            const int64_t ok = __shfl_xor((long long)key, d, 64);
            const int oi = __shfl_xor(id, d, 64);
            if (oi != 0x7fffffff && (id == 0x7fffffff || ok > key || (ok == key && oi < id))) {
                key = ok;
                id = oi;
            }
        }
        if ((id & 63) == lane) taken |= 1u << (id >> 6);
        const double l = logits[id];
        if (j == 0) top = l;
        if (lane == j) {
            my_id = id;
            my_logit = l;
        }
    }
    // (a NaN logit, infinite ones or a NaN in the inputs: every gate of the token is NaN, as the quotient gives)
    double sum = 0.0;
    bool nan = false;
    const double mine = lane < a.topk ? (double)expf((float)(my_logit - top)) : 0.0;
    for (int e = lane; e < a.E; e += 64) {
        const double l = logits[e];
        nan = nan || l != l;
        if (!a.renormalize) sum += (double)expf((float)(l - top));
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

template <int IN>
__global__ __launch_bounds__(kGateThreads) void moe_gate_kernel(const GateArgs a) {
    __shared__ double s_logit[kRouteMaxExperts];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t t = blockIdx.x;
    const char* const x = reinterpret_cast<const char*>(a.X) + t * a.H * 2;
    const int pieces = (int)((a.H + 15) / 16);
    for (int e = wave; e < a.E; e += kGateThreads / 64) {
        const char* const w = reinterpret_cast<const char*>(a.Wg) + e * a.H * 2;
        double l = 0.0;
        for (int p = lane; p < pieces; p += 64) {
            const W8Raw<IN> xr = load16<IN>(x, (int64_t)p * 16, a.H), wr = load16<IN>(w, (int64_t)p * 16, a.H);
#pragma unroll
            for (int i = 0; i < 16; ++i) l = fma((double)raw_value<IN>(xr, i), (double)raw_value<IN>(wr, i), l);
        }
#pragma unroll
        for (int d = 32; d >= 1; d >>= 1) l += __shfl_xor(l, d, 64);
        if (lane == 0) s_logit[e] = l;
    }
    __syncthreads();
    if (wave == 0) choose_experts(s_logit, t, a);
}

}  // namespace milo

using namespace milo;

extern "C" int milo_moe_route(const milo_half* X, int64_t T, int64_t H, const milo_half* Wg, int E, int topk, int n_shared, unsigned flags,
                              int32_t* ids, float* gates, void* stream) {
    if (!X || !Wg || !ids || !gates) return MILO_ERR_NULL;
    if (T < 1 || T > (int64_t(1) << 23) || H < 1 || H > (int64_t(1) << 20) || E < 1 || E > kRouteMaxExperts || topk < 1 || topk > E || topk > kRouteMaxTopk ||
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
    if (flags & MILO_ACT_BF16) moe_gate_kernel<W8_BF16><<<dim3((unsigned)T), dim3(kGateThreads), 0, (hipStream_t)stream>>>(a);
    else moe_gate_kernel<W8_F16><<<dim3((unsigned)T), dim3(kGateThreads), 0, (hipStream_t)stream>>>(a);
    return launch_status();
}
