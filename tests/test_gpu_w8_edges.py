"""The 8-bit path where its kernels could part from what is promised of them, against the 64-bit oracle (tolerances: see
test_gpu_w8.py; what a test adds to them is derived beside it)."""
import numpy as np
import pytest
import torch

import oracle
from test_gpu_w8 import DTYPES, U, V, check_layer, check_linear, f64, make_layer, normal, routing, unblock
from test_gpu_w8_kernels import kernel_of

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2504_02658_amd import api
    return api


# ---- the sum over a token's pairs --------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H", [1024, 1001])
def test_layer_of_many_pairs_adds_fp32_terms(api, H, dtype):
    # 16800 pairs, 68 MB of them: as exact as a layer of a few tokens
    T, F, E, topk = 2100, 64, 10, 8
    layer, host = make_layer(api, H, F, E, seed=15)
    X = normal(T, (T, H), dtype)
    ids, gates = routing(T, E, topk, seed=13)
    check_layer(layer.forward(X.cuda(), ids.cuda(), gates.cuda()), X, host, ids, gates)


@pytest.mark.parametrize("T", [1, 16, 40, 2100])
def test_layer_of_terms_beyond_fp16_that_cancel(api, T):
    # Expert 2i + 1 has the down projection of expert 2i with the other sign, and a gate that is a 64th smaller.  Terms of
    # up to some 10^6 leave a sum that fp16 holds.
    H, F, E, topk = 1024, 64, 8, 8
    host, dev = [], []
    for e in range(0, E, 2):
        W = [normal(e * 3 + i, s, torch.float32, std) for i, (s, std) in enumerate((((F, H), 0.05), ((F, H), 0.05), ((H, F), 6e3)))]
        for sign in (1.0, -1.0):
            ws = [W[0], W[1], W[2] * sign]
            host.append([oracle.quantize_rows(w.numpy()) for w in ws])
            dev.append(tuple(api.pack_w8(w.cuda()) for w in ws))
    X = normal(7, (T, H), torch.float16)
    ids = torch.stack([torch.randperm(E, generator=torch.Generator().manual_seed(t)) for t in range(T)]).to(torch.int32)
    gates = torch.where(ids % 2 == 0, 1.0, 1.0 - 2.0 ** -6).float()
    Y = api.W8MoELayer(dev, H, F).forward(X.cuda(), ids.cuda(), gates.cuda())
    ref, _, terms = oracle.w8a8_moe(X.float().numpy(), host, ids.numpy(), gates.numpy())
    assert terms.max() > 8 * 65504.0 and np.abs(ref).max() < 65504.0
    assert torch.isfinite(Y).all()
    check_layer(Y, X, host, ids, gates)


# ---- many experts ------------------------------------------------------------------------------------------------

def test_layer_of_more_experts_than_small_tiles_have_a_grid_for(api):
    # 8192 experts with 16384 features: 2^22 workgroups of 32 features and one slot's more.  (The experts share three sets of weights.)
    T, H, F, E = 17, 64, 16384, 8192
    some, hosts = make_layer(api, H, F, 3, seed=40)
    layer = api.W8MoELayer([some.experts[e % 3] for e in range(E)], H, F)
    X = normal(3, (T, H), torch.float16)
    ids = ((torch.arange(T) * 997 + 8191) % E).to(torch.int32).view(T, 1)
    gates = torch.rand((T, 1), generator=torch.Generator().manual_seed(1)) + 0.1
    assert len(set(ids.flatten().tolist())) == T and int(ids.max()) == E - 1
    Y = layer.forward(X.cuda(), ids.cuda(), gates.cuda())
    assert layer.routing_status() == 0
    check_layer(Y, X, hosts, ids % 3, gates)


# ---- the quantizer -----------------------------------------------------------------------------------------------

def test_pack_next_to_ties_at_the_smallest_scales(api):
    # scales of odd 24-bit numbers S in [2^-126, 2^-125): half of one is no fp32 number.  Units of 2^-149; values next to (n + 1/2) S.
    rng = np.random.default_rng(3)
    S = rng.integers(1 << 22, 1 << 23, 62) * 2 + 1
    S = np.concatenate([[15502097, (1 << 24) - 1], S]).astype(np.int64)
    rows = []
    for s in S:
        near = [(2 * n + 1) * s // 2 + d for n in range(0, 126) for d in (0, 1)]
        rows.append([127 * s] + near + [-v for v in near])
    W = (np.array(rows).astype(np.float64) * 2.0 ** -149).astype(np.float32)
    oc, os_ = oracle.quantize_rows(W)
    assert (os_ >= np.float32(2.0 ** -126)).all() and (os_ < np.float32(2.0 ** -125)).all()
    c, s = unblock(api.pack_w8(torch.from_numpy(W).cuda()).w8, *W.shape)
    assert np.array_equal(s, os_) and np.array_equal(c, oc)


# ---- SwiGLU rows -------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("T", [8, 16, 40, 700])
def test_layer_codes_of_swiglu_rows_at_ties(api, T):
    # x = (1, 0, 127, 0 ..), gate weights (32, 0, 0, 127 * 32), up weights (t, 0, 0, 127 t): codes (1, 0, 0, 127), so gate = 32,
    # SiLU(32) = 32 in fp32, up = t, and the SwiGLU row is 32 t, exactly.  It is 127 s and all (n + 1/2) s, with s no power of two.
    # The down projection copies it out: its codes show, and have to be those of the exact quotients, ties to even.
    H = F = 128
    S = [3, 5, 7, 11, 101, 333, 1021, 511]
    want, dev = [], []
    for s in S:
        h = np.concatenate([[127.0], np.arange(-63, 64) + 0.5]) * (s * 2.0 ** -9)
        t = torch.from_numpy(h / 32).float()
        W1, W3 = torch.zeros((F, H)), torch.zeros((F, H))
        W1[:, 0], W1[:, 3] = 32.0, 127.0 * 32.0
        W3[:, 0], W3[:, 3] = t, 127.0 * t
        assert np.array_equal(W3[:, 3].double().numpy(), 127.0 * h / 32)
        want.append(oracle.quantize_rows(h[None].astype(np.float32))[0][0])
        dev.append(tuple(api.pack_w8(w.cuda()) for w in (W1, W3, torch.eye(H))))
    X = torch.zeros((T, H), dtype=torch.bfloat16)
    X[:, 0], X[:, 2] = 1.0, 127.0
    ids = (torch.arange(T) % len(S)).to(torch.int32).view(T, 1)
    Y = f64(api.W8MoELayer(dev, H, F).forward(X.cuda(), ids.cuda(), torch.ones((T, 1)).cuda()))
    for t in range(T):
        got = Y[t] / (S[t % len(S)] * 2.0 ** -9)            # (the output's rounding: at most 127 * 2^-8 < 1/2)
        assert np.array_equal(np.rint(got), want[t % len(S)]), (t, S[t % len(S)])


@pytest.mark.parametrize("dtype", DTYPES)
def test_layer_results_do_not_depend_on_the_other_tokens(api, dtype):
    # One token alone, 13, 45 and 2100 of them take different kernels.  Codes are the same in all; a term carries at most five roundings of fp32, the
    # sum of eight seven more: 12 v of the terms' magnitudes on either side, and the output's rounding.
    T, H, F, E, topk = 2100, 1001, 300, 10, 8
    layer, host = make_layer(api, H, F, E, seed=25)
    X = normal(25, (T, H), dtype)
    ids, gates = routing(T, E, topk, seed=26)
    run = lambda rows: f64(layer.forward(X[rows].contiguous().cuda(), ids[rows].contiguous().cuda(), gates[rows].contiguous().cuda()))
    whole = run(slice(0, T))
    for first, n in ((0, 1), (2099, 1), (700, 13), (40, 16), (1000, 45), (1500, 300)):
        rows = slice(first, first + n)
        part = run(rows)
        terms = oracle.w8a8_moe(X[rows].float().numpy(), host, ids[rows].numpy(), gates[rows].numpy())[2]
        # (a rounding may fall on either side of a border: one step, 2 u, of the larger)
        tol = 24 * V * terms + 2 * U[dtype] * (np.maximum(np.abs(part), np.abs(whole[rows])) + 24 * V * terms) + 2.0 ** -24
        assert (np.abs(part - whole[rows]) <= tol).all()
        # (sums that far apart round to other outputs with the probability 24 v / 2 u of the terms over the output, fp16 0.2 % of some three)
        assert (part != whole[rows]).mean() < 0.02


@pytest.mark.parametrize("T", [2, 20, 300])
def test_layer_down_sums_that_cancel(api, T):
    # The second half of the features is the first half with the down projection's sign turned: every integer sum is zero, whatever
    # pieces of it the waves add up.  (Pieces added in 64 bits leave less than 2^-48 of their magnitude.)
    H, D = 64, 2560
    W1, W3, W2 = normal(1, (D, H), std=0.2), normal(2, (D, H), std=0.2), normal(3, (H, D), std=0.2)
    pack = lambda *ws: tuple(api.pack_w8(w.cuda()) for w in ws)
    two, one = pack(torch.cat([W1, W1]), torch.cat([W3, W3]), torch.cat([W2, -W2], 1)), pack(torch.cat([W1, W1]), torch.cat([W3, W3]), torch.cat([W2, 0 * W2], 1))
    X = normal(T, (T, H), torch.bfloat16).cuda()
    ids, gates = torch.zeros((T, 1), dtype=torch.int32, device="cuda"), torch.rand((T, 1), device="cuda") + 0.5
    half = f64(api.W8MoELayer([one], H, 2 * D).forward(X, ids, gates))
    Y = f64(api.W8MoELayer([two], H, 2 * D).forward(X, ids, gates))
    assert np.abs(half).max() > 1.0 and np.abs(Y).max() <= 2.0 ** -40 * np.abs(half).max()


# ---- long rows and large values ----------------------------------------------------------------------------------

@pytest.mark.parametrize("N,K,dtype", [(3, 65537, torch.float32), (17, 65600, torch.float16), (2, 131071, torch.bfloat16), (5, 131072, torch.float32),
                                       (1030, 65600, torch.float16), (1024, 66000, torch.bfloat16)])
def test_pack_of_rows_longer_than_the_registers_hold(api, N, K, dtype):
    # beyond 65536 columns a row is read twice; every code of varied rows, few rows and many
    W = normal(N + K, (N, K), dtype, 0.05)
    W[0, K - 1], W[N - 1, 65536] = 2.0, -3.0
    c, s = unblock(api.pack_w8(W.cuda()).w8, N, K)
    oc, os_ = oracle.quantize_rows(W.float().numpy())
    assert np.array_equal(c, oc) and np.array_equal(s, os_)


LONG = [("wide 16x16", 1, 20, 131072), ("wide 16x16", 9, 33, 70001), ("wide 16x32", 17, 20, 66000), ("wide 32x32", 17, 4000, 66000), ("wide 32x64", 40, 6000, 66000),
        ("wide 64x64", 70, 4000, 66000), ("tile 128x128", 260, 6000, 66000), ("tile 64x128", 400, 4000, 66000), ("tile 128x256", 520, 8000, 66000), ("wide 16x32", 1030, 20, 66000)]


@pytest.mark.parametrize("kernel,M,N,K", LONG)
def test_linear_of_long_varied_rows(api, kernel, M, N, K):
    # whole numbers below 2^53: the 64-bit product of the codes is exact wherever it runs, and in any order
    assert kernel_of(api, M, N, K) == kernel
    X, W = normal(M + K, (M, K), torch.bfloat16), normal(N + K, (N, K), torch.float16, 0.02)
    Y = api.w8a8_gemm(X.cuda(), api.pack_w8(W.cuda()))
    (xq, xs), (wq, ws) = oracle.quantize_rows(X.float().numpy()), oracle.quantize_rows(W.float().numpy())
    acc = torch.zeros((M, N), dtype=torch.float64, device="cuda")
    for k in range(0, K, 16384):
        acc += torch.from_numpy(xq[:, k:k + 16384]).cuda().double() @ torch.from_numpy(wq[:, k:k + 16384]).cuda().double().t()
    ref = acc.cpu().numpy() * xs.astype(np.float64)[:, None] * ws.astype(np.float64)[None, :]
    tol = np.abs(ref) * (U[torch.bfloat16] + 4 * V) + 1e-37
    assert (np.abs(f64(Y) - ref) <= tol).all()


@pytest.mark.parametrize("M", [1, 16, 200, 1100, 3000])
@pytest.mark.parametrize("K", [1, 100, 5000, 20000])
def test_rows_quantized_at_every_width_count_in_every_column(api, M, K):
    # two features whose weights vary over all columns
    X, W = normal(M + K, (M, K), torch.float16), normal(3 * K, (2, K), torch.float32)
    check_linear(api.w8a8_gemm(X.cuda(), api.pack_w8(W.cuda())), X, W)


@pytest.mark.parametrize("T", [2, 40, 300])
@pytest.mark.parametrize("H,F", [(70001, 48), (40, 70001), (64, 131072)])
def test_layer_of_long_rows(api, T, H, F):
    layer, host = make_layer(api, H, F, 2, seed=T + H, std=0.02)
    X = normal(T, (T, H), torch.float16, 0.2)
    ids, gates = routing(T, 2, 1, seed=T)
    check_layer(layer.forward(X.cuda(), ids.cuda(), gates.cuda()), X, host, ids, gates)


@pytest.mark.parametrize("M,N,K", [(1, 100, 4096), (16, 64, 14336), (40, 300, 1000), (300, 1000, 640), (2000, 4000, 300)])
def test_linear_of_the_largest_values(api, M, N, K):
    # K times the largest magnitude next to 2^120, brought back by the weights, one of whose rows is all of its largest value
    X, W = normal(M, (M, K), torch.float32), normal(N, (N, K), torch.float32)
    X = (X / X.abs().max() * (2.0 ** 120 / K * 0.99)).to(torch.bfloat16)
    X[0] = X.abs().max()
    W[0] = W.abs().max()
    W = W * 2.0 ** -100
    check_linear(api.w8a8_gemm(X.cuda(), api.pack_w8(W.cuda())), X, W)


# ---- router ------------------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("renormalize", [False, True])
@pytest.mark.parametrize("T,H,E,topk", [(3, 200, 40, 40), (33, 2048, 64, 6), (1100, 200, 40, 40), (1100, 2048, 64, 6), (1030, 64, 257, 64)])
def test_route_gates_are_rounded_once(api, T, H, E, topk, renormalize, dtype):
    # logits some tens to a hundred apart; exp, its sums and the quotient carry a few units of 2^-53, the logits' sums H of them
    # relative to their terms: below 2^-34 of a gate, so what counts is the rounding to fp32
    X, Wg = normal(T + H, (T, H), dtype), normal(E + H, (E, H), dtype, 20.0 / H ** 0.5)
    ids, gates = api.moe_route(X.cuda(), Wg.cuda(), topk, renormalize=renormalize)
    oi, og = oracle.moe_route(X.float().numpy(), Wg.float().numpy(), topk, renormalize, 0)
    assert np.array_equal(ids.cpu().numpy(), oi)
    assert (np.abs(gates.cpu().double().numpy() - og) <= og * V * (1 + 2.0 ** -9) + 2.0 ** -150).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T", [5, 1030])
def test_route_of_equal_sums_of_different_terms(api, T, dtype):
    # Experts in threes whose rows are each other's, permuted in pairs of columns that a token's activations do not tell apart: the sums are equal, their
    # terms come in another order, and all of them fit 53 bits.  Equal ones: the lowest id.
    H, E = 600, 30
    g = torch.Generator().manual_seed(T)
    X = torch.randint(-8, 9, (T, H // 2), generator=g).repeat(1, 2).to(dtype)
    W = torch.randint(-8, 9, (E // 3, H), generator=g)
    swap = torch.cat([W[:, H // 2:], W[:, :H // 2]], 1)
    half = torch.where(torch.arange(H) % (H // 2) % 2 == 0, W, swap)
    Wg = torch.stack([W, swap, half], 1).view(E, H).to(dtype)
    ids, _ = api.moe_route(X.cuda(), Wg.cuda(), 12)
    assert np.array_equal(ids.cpu().numpy(), oracle.moe_route(X.float().numpy(), Wg.float().numpy(), 12, True, 0)[0])
