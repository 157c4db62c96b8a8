"""Every kernel of the 8-bit path at sizes that reach it, against the 64-bit oracle (tolerances: see test_gpu_w8.py)."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from test_gpu_w8 import DTYPES, check_layer, check_linear, check_route, make_layer, normal, routing

pytestmark = pytest.mark.gpu

KERNELS = ["wide 16x16", "wide 16x32", "wide 16x64", "wide 32x32", "wide 32x64", "wide 64x64", "tile 64x128", "tile 128x128", "tile 128x256"]


@pytest.fixture(scope="module")
def api():
    from paper_2504_02658_amd import api
    return api


def kernel_of(api, M, N, K):
    f = api.lib().milo_w8a8_route
    f.argtypes = [ctypes.c_int64] * 3
    return KERNELS[f(M, N, K)]


LINEARS = [
    # few rows: features that end inside a workgroup's, K that ends inside a run of units or leaves waves idle
    ("wide 16x16", 1, 515, 8200), ("wide 16x16", 16, 48, 130), ("wide 16x32", 5, 6160, 700), ("wide 16x32", 16, 8203, 129),
    ("wide 16x64", 2, 12301, 320), ("wide 16x64", 16, 14336, 1408),
    # more rows
    ("wide 16x32", 70, 300, 1000), ("wide 16x32", 17, 17, 4100), ("wide 16x32", 252, 959, 307), ("wide 32x32", 272, 5740, 162), ("wide 32x32", 122, 1233, 3323),
    ("wide 32x64", 390, 4798, 137), ("wide 32x64", 125, 3266, 3622), ("wide 64x64", 300, 2000, 2050), ("wide 64x64", 99, 4973, 1315),
    # tiles: the last one with 1, 2, 31, 33 rows; features that are no multiple of eight; a few and many stages
    ("tile 64x128", 353, 4213, 130), ("tile 64x128", 1505, 929, 1074), ("tile 64x128", 2560, 736, 1725), ("tile 64x128", 258, 4744, 3224),
    ("tile 128x128", 1670, 5421, 386), ("tile 128x128", 2869, 1373, 1479), ("tile 128x128", 2079, 3880, 1003),
    ("tile 128x256", 2817, 5025, 138), ("tile 128x256", 1537, 3968, 666), ("tile 128x256", 1695, 3359, 1224), ("tile 128x256", 4097, 5000, 130), ("tile 128x256", 2079, 8200, 257),
]


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("kernel,M,N,K", LINEARS)
def test_linear_kernels(api, kernel, M, N, K, dtype):
    assert kernel_of(api, M, N, K) == kernel
    X, W = normal(M + K, (M, K), dtype), normal(N + K, (N, K), torch.float16, 0.02)
    w = api.pack_w8(W.cuda())
    flat = torch.full((M * N + 64,), 3.0, dtype=dtype, device="cuda")
    Y = api.w8a8_gemm(X.cuda(), w, out=flat[:M * N].view(M, N))
    assert (flat[M * N:] == 3.0).all()
    check_linear(Y, X, W)


@pytest.mark.parametrize("kernel,M,N,K", [c for c in LINEARS if c[0].startswith("tile")])
def test_tiles_count_their_waits(api, kernel, M, N, K):
    # the library in which every hand-counted wait is a wait for everything agrees bit for bit
    full = api.bind(api.FULLWAITS_LIB_PATH)
    X, w = normal(M, (M, K), torch.float16).cuda(), api.pack_w8(normal(N, (N, K)).cuda())
    Y = api.w8a8_gemm(X, w)
    assert torch.equal(Y, api._native.w8_gemm(full.entries, X, w.w8, N, K, None, None)) and (Y != 0).any()


@pytest.mark.parametrize("T,H,F", [(300, 128, 128), (500, 520, 1030), (260, 64, 4100), (300, 5000, 130), (260, 4500, 1030)])
def test_layer_tiles_count_their_waits(api, T, H, F):
    full = api.bind(api.FULLWAITS_LIB_PATH)
    layer, _ = make_layer(api, H, F, 3, seed=T)
    X = normal(T, (T, H), torch.bfloat16).cuda()
    ids, gates = (t.cuda() for t in routing(T, 3, 2, seed=T))
    Y = layer.forward(X, ids, gates)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    assert torch.equal(Y, api._native.w8_moe(full.entries, X, ids, gates, layer.table, H, F, 3, None, status, None)) and (Y != 0).any()


def test_linear_kernels_are_all_here():
    assert {k for k, *_ in LINEARS} == set(KERNELS)


@pytest.mark.parametrize("M", [1, 3, 16, 200, 1100, 3000])
@pytest.mark.parametrize("K", [1, 100, 5000, 20000])
def test_rows_quantized_at_every_width(api, M, K):
    # one output feature that copies column 0 back: code_x[m, 0] * 127 * scales, so the codes of X show
    X = normal(M + K, (M, K), torch.float16)
    W = torch.zeros((2, K), dtype=torch.float16)
    W[0, 0] = W[1, K - 1] = 1.0
    check_linear(api.w8a8_gemm(X.cuda(), api.pack_w8(W.cuda())), X, W)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,H,F,E,topk", [
    (300, 128, 128, 4, 2), (300, 130, 129, 4, 2), (260, 96, 500, 3, 1), (257, 520, 131, 2, 2), (900, 64, 258, 3, 3), (150, 72, 14400, 2, 1), (129, 40, 3, 1, 1),
    (100, 4096, 257, 16, 2), (17, 300, 520, 64, 8), (40, 513, 130, 30, 3),
    (300, 5000, 130, 3, 2), (260, 4502, 1030, 3, 2)])       # (tiles of 256 features in the down product: more than 128 of them)
def test_layer_kernels(api, T, H, F, E, topk, dtype):
    layer, host = make_layer(api, H, F, E, seed=T + H + F)
    X = normal(T, (T, H), dtype)
    ids, gates = routing(T, E, topk, seed=T * 7 + E)
    check_layer(layer.forward(X.cuda(), ids.cuda(), gates.cuda()), X, host, ids, gates)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,H,F,E,topk", [
    (9, 2100, 300, 8, 2), (16, 1030, 1100, 64, 8), (2, 9000, 130, 3, 2), (5, 200, 14500, 4, 2), (15, 2176, 4400, 5, 1), (4, 4096, 256, 6, 2), (4, 4097, 256, 6, 2)])
def test_layer_of_few_tokens_with_and_without_the_quantizer(api, T, H, F, E, topk, dtype):
    # codes of X and of the SwiGLU rows that the products form themselves, or that a launch of the quantizer does (16 and 64 KB)
    layer, host = make_layer(api, H, F, E, seed=T + H + F)
    X = normal(T, (T, H), dtype)
    ids, gates = routing(T, E, topk, seed=T * 5 + E)
    ids[T - 1, 0] = E
    check_layer(layer.forward(X.cuda(), ids.cuda(), gates.cuda()), X, host, ids, gates)
    assert layer.routing_status() == 6


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H", [1024, 1001])
def test_layer_of_many_pairs(api, H, dtype):
    # 16800 pairs: their outputs are kept in the activations' type, half a step of it more per term
    T, F, E, topk = 2100, 64, 10, 8
    layer, host = make_layer(api, H, F, E, seed=5)
    X = normal(T, (T, H), dtype)
    ids, gates = routing(T, E, topk, seed=3)
    ids[5, 2], ids[77] = 99, -1
    Y = layer.forward(X.cuda(), ids.cuda(), gates.cuda())
    assert layer.routing_status() == 6 and (Y[77] == 0).all()
    check_layer(Y, X, host, ids, gates, kept16=True)


@pytest.mark.parametrize("T", [4, 40, 700])
def test_layer_of_large_and_small_values(api, T):
    # SwiGLU rows far beyond fp16's range and far below it: what lies between the products has no 16-bit float's range.  (The down
    # projection's weights bring the outputs back.)
    H, F, E = 64, 200, 2
    for up, down in ((400.0, 1e-7), (1e-9, 3e4)):
        host, dev = [], []
        for e in range(E):
            ws = [normal(e * 3 + i, s, torch.float32, 0.3) * f for i, (s, f) in enumerate((((F, H), up), ((F, H), up), ((H, F), down)))]
            host.append([oracle.quantize_rows(w.numpy()) for w in ws])
            dev.append(tuple(api.pack_w8(w.cuda()) for w in ws))
        layer = api.W8MoELayer(dev, H, F)
        X = normal(T, (T, H), torch.bfloat16)
        ids, gates = routing(T, E, 2, seed=1)
        Y = layer.forward(X.cuda(), ids.cuda(), gates.cuda())
        ref, doubt, terms = oracle.w8a8_moe(X.float().numpy(), host, ids.numpy(), gates.numpy(), border=2.0 ** -8)        # (127 times the 2^-15 below)
        # a gate value of magnitude |a| enters the sigmoid with 3 steps of fp32, so SiLU(a) b carries up to |a| 2^-22: 2^-9 at 2^13
        # where the sigmoid is not yet 0 or 1 it is below 90: 2^-15
        d = doubt + terms * 2.0 ** -13
        tol = d + (np.abs(ref) + d) * 2.0 ** -8
        assert np.isfinite(ref).all() and (np.abs(Y.cpu().double().numpy() - ref) <= tol + 1e-37).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,H,E,topk", [(1025, 2048, 64, 6), (1040, 100, 16, 16), (1100, 333, 17, 4), (1200, 31, 256, 8), (1030, 64, 257, 8), (1500, 4100, 8, 2)])
def test_route_kernels(api, T, H, E, topk, dtype):
    check_route(api, normal(T + H, (T, H), dtype), normal(E, (E, H), dtype, 0.05), topk, True, 1)


@pytest.mark.parametrize("T", [1023, 1027])
def test_route_ties_and_nan_in_both_kernels(api, T):
    H, E = 96, 40
    X, Wg = normal(T, (T, H), torch.bfloat16), normal(3, (E, H), torch.bfloat16, 0.05)
    Wg[7] = Wg[30] = Wg[31] = Wg[2]
    X[0] = 0.0
    check_route(api, X, Wg, 12, False, 0)
    X[5, 3] = float("nan")
    ids, gates = (t.cpu() for t in api.moe_route(X.cuda(), Wg.cuda(), 5))
    assert ids[5].tolist() == [0, 1, 2, 3, 4] and torch.isnan(gates[5]).all() and torch.isfinite(gates[6:]).all()


def test_large_layer_captured_and_replayed(api):
    layer, _ = make_layer(api, 128, 256, 4, seed=9)
    T = 200
    X = torch.zeros((T, 128), dtype=torch.float16, device="cuda")
    ids, gates = (t.cuda() for t in routing(T, 4, 2, seed=1))
    layer.forward(X, ids, gates)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        Y = layer.forward(X, ids, gates)
    status = layer.last_status
    for i in range(4):
        X.copy_(normal(i, (T, 128), torch.float16))
        new = routing(T, 4, 2, seed=i)[0]
        if i == 2:
            new[3, 1] = 17
        ids.copy_(new)
        g.replay()
        torch.cuda.synchronize()
        assert int(status[0].item()) == (6 if i == 2 else 0)
        assert torch.equal(Y, layer.forward(X.clone(), ids.clone(), gates))
