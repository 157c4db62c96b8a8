"""The 8-bit oracle against closed forms, exact arithmetic and brute force, and the refusals of the 8-bit calls (all found on
the host before anything is launched, so they need no GPU)."""
import ctypes
from fractions import Fraction

import numpy as np
import pytest
import torch

import oracle
from paper_2504_02658_amd import api


def test_rows_of_hand():
    v = np.array([[127.0, -63.5, 0.5, 1.5, 2.5, 0.0], [0, 0, 0, 0, 0, 0], [-254.0, 1.0, 3.0, -1.0, 253.0, 2.0]], np.float32)
    q, s = oracle.quantize_rows(v)
    assert s.tolist() == [1.0, 0.0, 2.0]
    assert q.tolist() == [[127, -64, 0, 2, 2, 0], [0] * 6, [-127, 0, 2, 0, 126, 1]]      # halves go to the even code


def test_rows_against_exact_quotients():
    rng = np.random.default_rng(1)
    v = rng.standard_normal((3, 200)).astype(np.float32)
    q, s = oracle.quantize_rows(v)
    for r in range(3):
        for k in range(200):
            exact = Fraction(float(v[r, k])) / Fraction(float(s[r]))
            assert abs(exact - int(q[r, k])) <= Fraction(1, 2)
    assert (np.abs(q).max(1) == 127).all()


def test_rows_of_special_values():
    big = np.float32(3e38)
    v = np.array([[np.nan, 1], [np.inf, 1], [big, -big], [1e-37, -1e-38], [2.0 ** -119, 2.0 ** -120]], np.float32)
    q, s = oracle.quantize_rows(v)
    assert np.isnan(s[:2]).all() and (q[:2] == 0).all()
    assert q[2].tolist() == [127, -127]
    assert s[3] == 0 and (q[3] == 0).all()          # the scale would be subnormal
    assert s[4] >= 2.0 ** -126 and q[4, 0] == 127


def test_linear_is_the_product_of_what_codes_stand_for():
    rng = np.random.default_rng(2)
    W, X = rng.standard_normal((5, 70)).astype(np.float32), rng.standard_normal((3, 70)).astype(np.float32)
    c, s = oracle.quantize_rows(W)
    xq, xs = oracle.quantize_rows(X)
    Y = oracle.w8a8_linear(X, c, s)
    for m in range(3):
        for n in range(5):
            acc = sum(int(a) * int(b) for a, b in zip(xq[m], c[n]))
            assert Y[m, n] == acc * float(xs[m]) * float(s[n])


def test_route_of_hand():
    X = np.array([[1.0, 0.0], [0.0, 1.0], [0.0, 0.0]])
    Wg = np.array([[0.0, 2.0], [1.0, 2.0], [1.0, 0.0], [0.5, np.log(3)]])
    ids, gates = oracle.moe_route(X, Wg, 2, True, 1)
    assert ids.tolist() == [[1, 2, 4], [0, 1, 4], [0, 1, 4]]        # ties: the lowest id first
    assert np.allclose(gates, [[0.5, 0.5, 1]] * 3)
    p = np.exp(X @ Wg.T)
    p /= p.sum(1, keepdims=True)
    ids, gates = oracle.moe_route(X, Wg, 3, False, 0)
    assert np.allclose(gates, np.take_along_axis(p, ids.astype(int), 1))
    ids, gates = oracle.moe_route(np.array([[np.nan, 1.0]]), Wg, 2, True, 0)
    assert ids.tolist() == [[0, 1]] and np.isnan(gates).all()


def test_moe_is_chained_linears():
    rng = np.random.default_rng(3)
    H, F, E, T = 40, 24, 3, 4
    ws = [[oracle.quantize_rows(0.1 * rng.standard_normal(s).astype(np.float32)) for s in ((F, H), (F, H), (H, F))] for _ in range(E)]
    X = rng.standard_normal((T, H)).astype(np.float32)
    ids = np.array([[0, 2], [1, 0], [2, 7], [-1, 9]])
    gates = rng.random((T, 2)).astype(np.float32)
    Y, doubt, terms = oracle.w8a8_moe(X, ws, ids, gates)
    want = np.zeros((T, H))
    for t in range(T):
        for j in range(2):
            if not 0 <= ids[t, j] < E:
                continue
            w1, w3, w2 = ws[ids[t, j]]
            a, b = oracle.w8a8_linear(X[t:t + 1], *w1), oracle.w8a8_linear(X[t:t + 1], *w3)
            h = oracle.silu(a) * b
            step = np.abs(h).max() / 127
            want[t] += gates[t, j] * (step * np.rint(h / step) @ (w2[0].astype(float) * w2[1][:, None].astype(float)).T)[0]
    assert np.allclose(Y, want, rtol=1e-12, atol=1e-15) and (Y[3] == 0).all()
    assert (doubt == 0).all() and (terms >= np.abs(Y) - 1e-12).all()


# ---- sizes and refusals of the library ---------------------------------------------------------------------

@pytest.fixture(scope="module")
def L():
    return api.lib()


def test_sizes_whose_grids_fit(L):
    # 2^36 numbers at most: padded to 2^22 rows, more of them would need 2^32 threads of the quantizer
    for N, K in (((1 << 22) - 1, 1 << 14), (1 << 19, 1 << 17)):
        assert L.milo_w8_packed_bytes(N, K) > 0 and L.milo_w8a8_gemm_workspace(N, 1, K) > 0
        assert L.milo_w8_packed_bytes(N, K + 1) == 0 and L.milo_w8a8_gemm_workspace(N, 1, K + 1) == 0


def test_sizes(L):
    assert L.milo_w8_packed_bytes(16, 128) == 16 * 128 + 64
    assert L.milo_w8_packed_bytes(1, 1) == 16 * 128 + 64
    assert L.milo_w8_packed_bytes(17, 129) == 32 * 256 + 128
    assert L.milo_w8_packed_bytes(14336, 4096) == 14336 * 4096 + 14336 * 4
    for N, K in ((0, 64), (64, 0), (-1, 64), (16, (1 << 17) + 1), (1 << 22, 16)):
        assert L.milo_w8_packed_bytes(N, K) == 0
    assert L.milo_w8a8_gemm_workspace(1, 64, 128) >= 16 * 128 + 64
    assert L.milo_w8a8_gemm_workspace(0, 64, 128) == 0 and L.milo_w8a8_gemm_workspace(4, 0, 128) == 0
    assert L.milo_w8a8_gemm_workspace(1 << 22, 64, 128) == 0 and L.milo_w8a8_gemm_workspace((1 << 22) - 1, 64, 128) > 0
    assert L.milo_w8a8_gemm_workspace(1 << 19, (1 << 17) + 1, 128) == 0 and L.milo_w8a8_gemm_workspace(1 << 19, 1 << 17, 128) > 0     # M N
    assert L.milo_moe_w8a8_workspace(4, 128, 256, 8, 2) > 0
    assert L.milo_moe_w8a8_workspace(512, 4096, 14336, 8, 2) >= 512 * 2 * 14336
    for bad in ((0, 128, 256, 8, 2), (4, 0, 256, 8, 2), (4, 128, 0, 8, 2), (4, 128, 256, 0, 1), (4, 128, 256, 8, 0), (4, 128, 256, 8, 9),
                (1 << 23, 4096, 4096, 8, 2), (1 << 23, 1, 1, 8, 1), (4, 128, 256, 65537, 2), (4, 64, 1 << 15, 1 << 13, 2)):
        assert L.milo_moe_w8a8_workspace(*bad) == 0


P, ODD = ctypes.c_void_p(0x10000), ctypes.c_void_p(0x10008)


def test_pack_refuses(L):
    ok = [P, 0, 32, 64, P, None]
    for i, v, status in ((0, None, 1), (4, None, 1), (1, 3, 2), (1, -1, 2), (2, 0, 2), (3, 0, 2), (3, (1 << 17) + 1, 2), (0, ODD, 7), (4, ODD, 7)):
        a = list(ok)
        a[i] = v
        assert L.milo_pack_w8(*a) == status, (i, v)


def test_linear_refuses(L):
    need = L.milo_w8a8_gemm_workspace(4, 32, 64)
    ok = [P, 4, 32, 64, P, 0, P, P, need, None]
    for i, v, status in ((0, None, 1), (4, None, 1), (6, None, 1), (1, 0, 2), (1, 1 << 22, 2), (2, 0, 2), (3, -4, 2), (5, 1, 2), (5, 2, 2), (7, None, 5),
                         (8, need - 1, 5), (0, ODD, 7), (4, ODD, 7), (6, ODD, 7), (7, ODD, 7)):
        a = list(ok)
        a[i] = v
        assert L.milo_w8a8_gemm(*a) == status, (i, v)


def test_route_refuses(L):
    ok = [P, 4, 64, P, 8, 2, 1, 0, P, P, None]
    for i, v, status in ((0, None, 1), (3, None, 1), (8, None, 1), (9, None, 1), (1, 0, 2), (1, 1 << 22, 2), (2, 0, 2), (2, (1 << 20) + 1, 2), (4, 0, 2), (4, 1025, 2), (5, 0, 2), (5, 9, 2), (6, -1, 2),
                         (6, 65, 2), (7, 1, 2), (7, 16, 2), (0, ODD, 7), (3, ODD, 7), (8, ODD, 7), (9, ODD, 7)):
        a = list(ok)
        a[i] = v
        assert L.milo_moe_route(*a) == status, (i, v)
    assert L.milo_moe_route(P, 4, 64, P, 128, 65, 0, 0, P, P, None) == 2


def test_layer_refuses(L):
    need = L.milo_moe_w8a8_workspace(4, 64, 96, 8, 2)
    ok = [P, 4, 64, 96, P, 8, P, P, 2, 0, P, P, P, need, None]
    for i, v, status in ((0, None, 1), (4, None, 1), (6, None, 1), (7, None, 1), (10, None, 1), (1, 0, 2), (2, 0, 2), (3, 0, 2), (5, 0, 2), (8, 0, 2), (8, 9, 2),
                         (9, 1, 2), (12, None, 5), (13, need - 1, 5), (0, ODD, 7), (4, ODD, 7), (6, ODD, 7), (7, ODD, 7), (10, ODD, 7), (11, ODD, 7), (12, ODD, 7)):
        a = list(ok)
        a[i] = v
        assert L.milo_moe_w8a8_forward(*a) == status, (i, v)
    t = (api.W8Expert * 2)(api.W8Expert(16, 32, 48), api.W8Expert(16, 32, 48))
    assert L.milo_moe_w8a8_check_experts(t, 2, 64, 96) == 0
    assert L.milo_moe_w8a8_check_experts(None, 2, 64, 96) == 1
    assert L.milo_moe_w8a8_check_experts(t, 0, 64, 96) == 2 and L.milo_moe_w8a8_check_experts(t, 2, 0, 96) == 2
    t[1].w3 = 0
    assert L.milo_moe_w8a8_check_experts(t, 2, 64, 96) == 1
    t[1].w3 = 8
    assert L.milo_moe_w8a8_check_experts(t, 2, 64, 96) == 7


def test_python_calls_refuse_host_tensors():
    w = api.W8Weight(16, 64, torch.zeros(16 * 128 + 64, dtype=torch.uint8))
    with pytest.raises(TypeError):
        api.pack_w8(torch.zeros(16, 64))
    with pytest.raises(TypeError):
        api.w8a8_gemm(torch.zeros(1, 64, dtype=torch.float16), w)
    with pytest.raises(TypeError):
        api.moe_route(torch.zeros(1, 64, dtype=torch.float16), torch.zeros(4, 64, dtype=torch.float16), 2)
    with pytest.raises(ValueError):
        api.W8MoELayer([(w, w, w)], 64, 32)
