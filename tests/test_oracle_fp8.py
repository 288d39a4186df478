"""Pins of the oracle's 8-bit layers: e4m3 from the format's arithmetic, hand-worked blocks, brute-force products."""
import numpy as np
import torch

import oracle


def _all_values():
    """Every finite e4m3 value by the format's arithmetic, by code 0 .. 126 (non-negative)."""
    vals = []
    for code in range(127):
        e, m = code >> 3, code & 7
        vals.append(m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(vals)


def test_e4m3_values_are_fixed_points_and_midpoints_go_to_the_even_code():
    v = _all_values()
    assert v[-1] == 448.0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6
    assert np.array_equal(oracle.e4m3_round(v), v) and np.array_equal(oracle.e4m3_round(-v), -v)
    mid = (v[:-1] + v[1:]) / 2
    want = np.where(np.arange(len(mid)) % 2 == 0, v[:-1], v[1:])
    assert np.array_equal(oracle.e4m3_round(mid), want)
    assert np.array_equal(oracle.e4m3_round(np.nextafter(mid, 1e9)), v[1:])
    assert np.array_equal(oracle.e4m3_round(np.nextafter(mid, 0)), v[:-1])
    assert np.all(oracle.e4m3_round(np.array([460.0, 1e9, -500.0])) == [448.0, 448.0, -448.0])


def test_e4m3_round_agrees_with_torch():
    rng = np.random.default_rng(0)
    v = (rng.standard_normal(20000) * 10.0 ** rng.uniform(-4, 2, 20000)).astype(np.float32)
    v = v[np.abs(v) <= 448]
    t = torch.from_numpy(v).to(torch.float8_e4m3fn).to(torch.float32).numpy()
    assert np.array_equal(oracle.e4m3_round(v), t)


def test_blocks_by_hand():
    v = np.zeros((2, 130))
    v[0, 0], v[0, 5], v[0, 129] = 896.0, -3.0, 7.0       # first group: scale 2; second: scale 7 / 448 = 1 / 64
    q, s = oracle.fp8_quotients(v)
    assert q.shape == (2, 256) and s.shape == (2, 2)
    assert list(s[0]) == [2.0, 1 / 64] and list(s[1]) == [1.0, 1.0]
    assert q[0, 0] == 448 and q[0, 5] == -1.5 and q[0, 129] == 448 and not q[0, 130:].any() and not q[1].any()
    assert oracle.fp8_quotients(np.full((1, 3), 1e-45))[1][0, 0] == 2.0 ** -126
    w = np.zeros((129, 128))
    w[127, 3], w[128, 0] = 448.0, 4.48
    q, s = oracle.fp8_quotients_weights(w)
    assert s.shape == (2, 1) and s[0, 0] == 1.0 and abs(s[1, 0] - 0.01) < 1e-15 and q.shape == (129, 128)
    assert q[127, 3] == 448 and abs(q[128, 0] - 448) < 1e-9


def test_rmsnorm_by_hand():
    h = np.array([[3.0, -4.0, 0.0, 0.0], [0.0, 0.0, 0.0, 0.0]])
    w = np.array([1.0, 2.0, 3.0, 4.0])
    assert np.allclose(oracle.rmsnorm(h, w, 0.0), [[1.2, -3.2, 0, 0], [0, 0, 0, 0]])
    assert np.allclose(oracle.rmsnorm(h, w, 2.75)[0], [1.0, -8 / 3, 0, 0])      # mean 6.25 + 2.75 = 9


def test_gemm_against_loops():
    rng = np.random.default_rng(1)
    T, K, N = 3, 256, 130
    qx, qw = oracle.e4m3_round(rng.standard_normal((T, K)) * 100), oracle.e4m3_round(rng.standard_normal((N, K)) * 100)
    sx, sw = rng.uniform(0.1, 2, (T, 2)), rng.uniform(0.1, 2, (2, 2))
    y, mag = oracle.gemm_fp8(qx, sx, qw, sw)
    for t in range(T):
        for n in (0, 127, 128, 129):
            terms = [sx[t, k // 128] * sw[n // 128, k // 128] * qx[t, k] * qw[n, k] for k in range(K)]
            assert abs(y[t, n] - sum(terms)) < 1e-9 * mag[t, n] and abs(mag[t, n] - sum(abs(x) for x in terms)) < 1e-9 * mag[t, n]


def test_gated_by_hand():
    assert oracle.gated(np.array([0.0]), np.array([5.0]))[0] == 0.0
    assert abs(oracle.gated(np.array([np.log(3.0)]), np.array([4.0]))[0] - 3.0 * np.log(3.0)) < 1e-12      # 1 / (1 + 1/3) = 3/4
    assert oracle.gated(np.array([-1000.0]), np.array([1.0]))[0] == 0.0
