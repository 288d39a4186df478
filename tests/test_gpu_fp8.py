"""GPU parity of the 8-bit layers against the CPU oracle.

Tolerances, u = 2^-24 the half step of fp32:
  scales        amax / 448 with one correction step: 4 u; behind a norm DELTA more (below).
  codes         a code is the e4m3 value nearest to the computed quotient: |code - quotient| <= half the step there plus the quotient's
                own error, 8 u (the scale, its reciprocal with one correction step, one product).
  norm          v = h pre rms w: the sum of squares is a chain of at most 8 chunks * 8 values * rounds a lane and 12 joins, each within u
                and all terms positive, halved by the root; root, division, mean, three products: 10 u more.
  products      exact terms.  The matrix instruction adds the products of eight consecutive codes on the grid of 13 bits below the
                largest exponent among them (test_matrix_instruction_adds_runs_of_eight_on_a_grid pins it): seven of them lose less than a
                step each, 7 * 2^-13 max |term| of every run, counted for its products alone; further additions, 16 in the instruction and
                one of K / 128 in fp32, each within 2^-23 of the terms' magnitudes (a truncating adder counted in; 128 for the plain kernel,
                which adds one product at a time): (128 + K / 128 + 4) 2^-23 sum |terms|; one rounding to bf16, 2^-8.
  gated         |silu'| <= 1.1 and |silu(g)| <= |g|: errors of both products through them, 8 u of exp, division and product; bf16.
"""
import numpy as np
import pytest
import torch

import oracle
import paper_2503_17513_amd as pme

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
EPS = 1e-5


@pytest.fixture(autouse=True)
def _reset():
    yield
    pme.set_path(pme.PATH_AUTO)
    pme.set_gemm_tile(0)


def _rand(shape, seed, outliers=True, dtype=torch.bfloat16):
    rng = np.random.default_rng(seed)
    x = rng.standard_normal(shape)
    if outliers:
        x[:, rng.integers(0, shape[1], max(1, shape[1] // 100))] *= 50.0
    return torch.from_numpy(x.astype(np.float32)).to(dtype).cuda()


def _f64(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _codes64(q):
    return q.detach().cpu().to(torch.float32).numpy().astype(np.float64)


def check_codes(q, s, quotient, scale, delta):
    """Codes and scales against the oracle's quotients (before rounding) and scales."""
    s, q = _f64(s), _codes64(q)
    assert s.shape == scale.shape and q.shape == quotient.shape
    rel = np.abs(s - scale) / scale
    assert rel.max(initial=0) <= delta + 4 * U, f"scale off by {rel.max():.3e}"
    err = np.abs(q - quotient) - oracle.e4m3_step(quotient) / 2
    assert np.all(err <= (2 * delta + 8 * U) * np.abs(quotient)), f"code off by {err.max():.3e} more than half a step"
    assert np.array_equal(q, oracle.e4m3_round(q))


def norm_delta(d):
    chunks = max(1, -(-d // 8) // 64)                # a lane's chunks, at most (rows on one wave)
    return ((8 * chunks + 12) / 2 + 10) * U


# ---- norm, residual, codes

NORM_CASES = [
    # T, d, type, weight type, residual
    (1, 2048, "bf16", "bf16", True), (1, 1, "bf16", "bf16", True), (2, 7, "f32", "f32", False), (3, 127, "bf16", "f32", True),
    (3, 128, "f32", "bf16", True), (5, 129, "bf16", "bf16", False), (4, 2000, "f32", "f32", True), (9, 4096, "bf16", "bf16", True),
    (2, 14336, "bf16", "bf16", True), (3, 16387, "f32", "f32", True), (2, 32768, "bf16", "bf16", False), (2, 40001, "bf16", "f32", True), (1, 70000, "f32", "f32", True),
    (1, 1 << 20, "bf16", "bf16", False), (513, 2048, "bf16", "bf16", True), (600, 1999, "bf16", "bf16", True), (700, 130, "f32", "f32", False),
    (521, 4096, "bf16", "bf16", True), (515, 8200, "f32", "bf16", False),
]
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.mark.parametrize("T,d,xt,wt,residual", NORM_CASES)
def test_rmsnorm_quant(T, d, xt, wt, residual):
    x = _rand((T, d), d + T, dtype=DT[xt])
    w = _rand((1, d), d, outliers=False, dtype=DT[wt])[0]
    r = _rand((T, d), d + T + 1, outliers=False, dtype=DT[xt]) if residual else None
    if T > 2:
        x[1] = 0
        if residual:
            r[1] = 0
    out = pme.rmsnorm_quant_fp8(x, w, EPS, r)
    torch.cuda.synchronize()
    h = (x.float() + r.float()).to(DT[xt]) if residual else x
    if residual:
        assert torch.equal(out[2], h)                 # one addition and one rounding
    quotient, scale = oracle.fp8_quotients(oracle.rmsnorm(_f64(h), _f64(w), EPS))
    check_codes(out[0], out[1], quotient, scale, norm_delta(d))
    if T > 2:
        assert not _codes64(out[0])[1].any() and bool((out[1][1] == 1).all())


def test_rmsnorm_in_place_pitches_and_odd_addresses():
    T, d = 37, 1003
    for xt in ("bf16", "f32"):
        w = _rand((1, d), 5, outliers=False, dtype=DT[xt])[0]
        big = [_rand((T, d + 30), 6 + i, dtype=DT[xt]) for i in range(3)]
        x, r, h = big[0][:, 1:1 + d], big[1][:, 3:3 + d], big[2][:, 17:17 + d]       # odd pitches and odd first columns
        want = (x.float() + r.float()).to(DT[xt])
        around = [b.clone() for b in big]
        quotient, scale = oracle.fp8_quotients(oracle.rmsnorm(_f64(want), _f64(w), EPS))
        q, s, got = pme.rmsnorm_quant_fp8(x, w, EPS, r, h)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and got.data_ptr() == h.data_ptr()
        check_codes(q, s, quotient, scale, norm_delta(d))
        around[2][:, 17:17 + d] = want                # nothing beside the rows has changed
        assert all(torch.equal(a, b) for a, b in zip(around, big))
        for alias in (x, r):                          # the stream updated in place
            xa, ra = x.clone(), r.clone()
            dst = xa if alias is x else ra
            q2, s2, h2 = pme.rmsnorm_quant_fp8(xa, w, EPS, ra, dst)
            torch.cuda.synchronize()
            assert torch.equal(h2, want) and torch.equal(q2.view(torch.uint8), q.view(torch.uint8)) and torch.equal(s2, s)


@pytest.mark.parametrize("d", [256, 5000, 40000])
def test_rmsnorm_rows_beyond_the_squares_range(d):
    """Squares that overflow or vanish in fp32, eps of zero, zeros, values that are not finite: each row by itself."""
    x = _rand((8, d), 3, dtype=torch.float32)
    for i, f in enumerate((1e30, 1e-30, 1e-42, 1.0, 1e36)):
        x[i] *= f
    x[5] = 0
    x[6, d // 2] = float("nan")
    x[7, d - 1] = float("-inf")
    w = _rand((1, d), 4, outliers=False, dtype=torch.float32)[0]
    for eps in (0.0, 1e-30, 1e-5):
        q, s = pme.rmsnorm_quant_fp8(x, w, eps)
        torch.cuda.synchronize()
        quotient, scale = oracle.fp8_quotients(oracle.rmsnorm(_f64(x[:6]), _f64(w), np.float32(eps)))
        # behind eps = 1e-5 the row of subnormal values stays subnormal, which is not within half a step of fp32's relative rounding
        keep = [0, 1, 2, 3, 4, 5] if eps < 1e-20 else [0, 1, 3, 4, 5]
        check_codes(q[keep], s[keep], quotient[keep], scale[keep], norm_delta(d) + 4 * U)
        assert bool(torch.isnan(q[6:].float()).all()) and bool(torch.isnan(s[6:]).all())


@pytest.mark.parametrize("d", [1, 256, 5000, 40000])
def test_rmsnorm_mean_and_eps_that_overflow_together(d):
    """Squares whose sum fits fp32 and an eps that fits it, while the mean and eps together do not (the last row: they do)."""
    x = _rand((4, d), 13, dtype=torch.float32)
    x /= x.norm(dim=1, keepdim=True)
    for i, f in enumerate((1.8e19, 1e19, 5e17, 1.0)):   # FLT_MAX is 3.4028e38, the spacing below it 2e31
        x[i] *= f
    w = _rand((1, d), 14, outliers=False, dtype=torch.float32)[0]
    for eps in (3.4028234e38, 3.4e38, 3e38):
        q, s = pme.rmsnorm_quant_fp8(x, w, eps)
        torch.cuda.synchronize()
        quotient, scale = oracle.fp8_quotients(oracle.rmsnorm(_f64(x), _f64(w), np.float32(eps)))
        check_codes(q, s, quotient, scale, norm_delta(d) + 4 * U)


# ---- quantizers

@pytest.mark.parametrize("T,d,xt", [(1, 1, "bf16"), (3, 130, "f32"), (8, 8192, "bf16"), (5, 1999, "bf16"), (2, 40001, "f32"), (1100, 4096, "bf16"), (333, 14336, "f32"), (1, 1 << 20, "bf16")])
def test_quant(T, d, xt):
    x = _rand((T, d), d, dtype=DT[xt])
    if T > 2:
        x[1] = 0
    q, s = pme.quant_fp8(x)
    torch.cuda.synchronize()
    check_codes(q, s, *oracle.fp8_quotients(_f64(x)), 0.0)


def test_quant_extremes():
    x = torch.zeros((7, 200), dtype=torch.float32, device="cuda")
    x[0, 3], x[1, 150], x[2, 0], x[3, 5] = 3.4e38, 1e-40, float("inf"), float("nan")
    x[4, 7], x[4, 8] = -1e-30, 3e-33
    x[5, :128], x[6, 199] = 2.0, -0.0
    q, s = pme.quant_fp8(x)
    torch.cuda.synchronize()
    ok = [0, 1, 4, 5, 6]
    check_codes(q[ok], s[ok], *oracle.fp8_quotients(_f64(x[ok])), 0.0)
    assert s[1, 1] == 2.0 ** -126
    for row in (2, 3):
        assert bool(torch.isnan(s[row, 0])) and bool(torch.isnan(q[row, :128].float()).all()) and s[row, 1] == 1 and not bool(q[row, 128:].float().any())


def test_codes_beyond_the_row():
    """0, or NaN where their block's scale is NaN: the product is NaN for that token, and whole for the others."""
    x = _rand((5, 200), 9, dtype=torch.float32)
    x[1, 150], x[2, 3], x[3, 199] = float("inf"), float("nan"), float("nan")
    w = _rand((1, 200), 10, outliers=False, dtype=torch.float32)[0]
    for q, s, blocks in ((*pme.quant_fp8(x), [(1, 1), (2, 0), (3, 1)]), (*pme.rmsnorm_quant_fp8(x, w, EPS), [(t, b) for t in (1, 2, 3) for b in (0, 1)])):
        bad = torch.zeros((5, 2), dtype=torch.bool, device="cuda")
        for t, b in blocks:
            bad[t, b] = True
        y = pme.fp8_gemm(q, s, torch.ones((8, 256), device="cuda").to(q.dtype), torch.ones((1, 2), device="cuda"))
        torch.cuda.synchronize()
        assert torch.equal(torch.isnan(s), bad) and torch.equal(torch.isnan(q.float()).view(5, 2, 128).all(2), bad)
        assert torch.equal(torch.isnan(q.float()).view(5, 2, 128).any(2), bad)
        assert not bool(q[[0, 4], 200:].float().any()) and torch.equal(torch.isnan(y), bad.any(1, keepdim=True).expand(5, 8))


def test_quant_pitch_and_odd_address():
    big = _rand((19, 700), 2)
    x = big[:, 5:5 + 301]
    q, s = pme.quant_fp8(x)
    torch.cuda.synchronize()
    check_codes(q, s, *oracle.fp8_quotients(_f64(x)), 0.0)


@pytest.mark.parametrize("xt", ["bf16", "f32"])
def test_codes_are_nearest_to_quotients_by_the_stored_scale(xt):
    """Half a step and 2^-22 of the exact quotient by the scale that is returned: the reciprocal is rounded once behind a correction of its
    square, and so is the product, 2 2^-24 and less than 2^-44 (twice that allowed)."""
    x = _rand((700, 4096), 31, dtype=DT[xt])
    for f, per in ((pme.quant_fp8, 1), (pme.quantize_weights_fp8, 128)):
        q, s = f(x)
        torch.cuda.synchronize()
        quotient = _f64(x) / np.repeat(np.repeat(_f64(s), per, axis=0)[:700], 128, axis=1)
        err = np.abs(_codes64(q) - np.clip(quotient, -448.0, 448.0)) - oracle.e4m3_step(quotient) / 2
        assert np.all(err <= 2.0 ** -22 * np.abs(quotient)), err.max()


def test_midpoints_go_to_the_even_code():
    """Scales that are powers of two: all midpoints of neighbouring codes, their neighbours in fp32, and what lies below the smallest code."""
    v = np.unique(np.abs(torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()))
    v = v[np.isfinite(v)].astype(np.float64)
    assert len(v) == 127 and v[-1] == 448
    mid = ((v[1:] + v[:-1]) / 2).astype(np.float32)
    row = np.concatenate([mid, np.nextafter(mid, np.float32(0)), np.nextafter(mid, np.float32(1e9)), v[:-1].astype(np.float32), np.float32([1e-6, 2.0 ** -149, -0.0])])
    row = np.concatenate([row, -row, np.zeros(-2 * len(row) % 127, np.float32)]).reshape(-1, 127)
    row = np.concatenate([row, np.full((len(row), 1), 448.0, np.float32)], axis=1)          # every block's scale is 1
    for p in (-20, 0, 33):
        x = torch.from_numpy(np.ldexp(row, p)).cuda()
        for q, s in (pme.quant_fp8(x), pme.quantize_weights_fp8(x)):
            torch.cuda.synchronize()
            assert bool((s == 2.0 ** p).all())
            assert np.array_equal(_codes64(q), oracle.e4m3_round(np.ldexp(np.ldexp(row, p).astype(np.float64), -p)))


@pytest.mark.parametrize("N,d,xt", [(1, 1, "bf16"), (127, 130, "f32"), (128, 128, "bf16"), (129, 2000, "bf16"), (300, 1024, "f32"), (2048, 257, "bf16")])
def test_quantize_weights(N, d, xt):
    w = _rand((N, d + 3), N + d, dtype=DT[xt])[:, 1:1 + d]
    if N > 256:
        w[128:256] = 0
    q, s = pme.quantize_weights_fp8(w)
    torch.cuda.synchronize()
    check_codes(q, s, *oracle.fp8_quotients_weights(_f64(w)), 0.0)


# ---- products

def _operands(T, K, N, seed, mats=1):
    """Codes of heavy-tailed activations and Gaussian weights by the oracle's quantizer, on the device."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((T, K))
    x[:, rng.integers(0, K, max(1, K // 100))] *= 50.0
    out = []
    for v, f in [(x, oracle.fp8_quotients)] + [(rng.standard_normal((N, K)), oracle.fp8_quotients_weights) for _ in range(mats)]:
        quotient, s = f(v)
        q = oracle.e4m3_round(quotient).astype(np.float32)
        out += [torch.from_numpy(q).cuda().to(torch.float8_e4m3fn), torch.from_numpy(s.astype(np.float32)).cuda()]
    return out


def _products(ops):
    qx, sx = _codes64(ops[0]), _f64(ops[1])
    return [oracle.gemm_fp8(qx, sx, _codes64(q), _f64(s)) for q, s in zip(ops[2::2], ops[3::2])]


def _sum_errors(ops, mags):
    """Bounds on the errors of the sums behind `mags`: additions in fp32, and the grid of the matrix instruction."""
    K = ops[0].shape[1]
    out = []
    x = np.abs(_codes64(ops[0]) * np.repeat(_f64(ops[1]), 128, axis=1))
    for (q, s), mag in zip(zip(ops[2::2], ops[3::2]), mags):
        w = np.abs(_codes64(q) * np.repeat(np.repeat(_f64(s), 128, axis=0)[: len(q)], 128, axis=1))
        runs = np.zeros_like(mag)
        for k in range(0, K, 8):
            best = np.zeros_like(mag)
            for e in range(k, k + 8):
                np.maximum(best, np.outer(x[:, e], w[:, e]), out=best)
            runs += best
        out.append(1.01 * ((128 + K / 128 + 4) * 2.0 ** -23 * mag + 7 * 2.0 ** -13 * runs))
    return out


def check_gemm(y, ops):
    (ref, mag), = _products(ops)
    err = np.abs(_f64(y) - ref)
    lim = 2.0 ** -8 * np.abs(ref) + 1.01 * _sum_errors(ops, [mag])[0]
    assert np.all(err <= lim), f"product off by {np.max(err / lim):.2f} times its bound"


def check_gated(y, ops):
    (g, gm), (u, um) = _products(ops)
    ref = oracle.gated(g, u)
    dg, du = _sum_errors(ops, [gm, um])
    lim = 2.0 ** -8 * np.abs(ref) + 1.01 * (1.1 * dg * np.abs(u) + np.abs(g) * du + 1.1 * dg * du + 8 * U * np.abs(ref))
    err = np.abs(_f64(y) - ref)
    assert np.all(err <= lim), f"gated product off by {np.max(err / lim):.2f} times its bound"


def test_matrix_instruction_adds_runs_of_eight_on_a_grid():
    """448 * 256 in one run of eight products and its negative in the next: what is left of a small product in the first run is what lies
    on the grid, 13 bits below the exponent 16 of the large one; in a run of its own all of it is left."""
    x, w = torch.zeros((1, 128), device="cuda"), torch.zeros((1, 128), device="cuda")
    x[0, 0], x[0, 8], w[0, 0], w[0, 8] = 448.0, -448.0, 256.0, 256.0
    one = torch.ones((1, 1), device="cuda")
    pme.set_path(pme.PATH_MFMA)
    for at, small, left in ((5, 8.0, 8.0), (7, 24.0, 24.0), (5, 4.0, 0.0), (3, -8.0, -8.0), (16, 4.0, 4.0), (127, 0.25, 0.25)):
        xs, ws = x.clone(), w.clone()
        xs[0, at], ws[0, at] = small, 1.0
        y = pme.fp8_gemm(xs.to(torch.float8_e4m3fn), one, ws.to(torch.float8_e4m3fn), one)
        torch.cuda.synchronize()
        assert float(y) == left, (at, small)


PATHS = (pme.PATH_GENERIC, pme.PATH_AUTO)
GEMM_SHAPES = [(1, 128, 1), (1, 256, 130), (3, 128, 64), (16, 384, 129), (17, 1024, 255), (33, 640, 300), (64, 2048, 256), (100, 1152, 131),
               (130, 512, 700), (257, 1280, 513)]


@pytest.mark.parametrize("T,K,N", GEMM_SHAPES)
def test_fp8_gemm(T, K, N):
    ops = _operands(T, K, N, T + K + N)
    for path in PATHS:
        pme.set_path(path)
        y = pme.fp8_gemm(*ops)
        torch.cuda.synchronize()
        check_gemm(y, ops)


@pytest.mark.parametrize("T,K,N", GEMM_SHAPES)
def test_fp8_gated_gemm(T, K, N):
    ops = _operands(T, K, N, T + K + N, mats=2)
    for path in PATHS:
        pme.set_path(path)
        y = pme.fp8_gated_gemm(*ops)
        torch.cuda.synchronize()
        check_gated(y, ops)


# every tile, forced: one K block and fewer blocks than waves, K blocks that fill neither a stage nor a group of four scales, uneven shares
# of K, rings filled several times, several tiles with ragged ends
TILES = range(201, 214)
TILE_SHAPES = [(1, 128, 16), (8, 384, 33), (40, 384, 72), (300, 640, 530), (257, 1152, 385), (96, 2432, 128), (7, 8320, 40), (33, 12416, 72), (16, 6144, 130)]


@pytest.mark.parametrize("T,K,N", TILE_SHAPES)
@pytest.mark.parametrize("tile", TILES)
def test_fp8_tiles(tile, T, K, N):
    ops = _operands(T, K, N, tile + T + K + N, mats=2)
    pme.set_path(pme.PATH_MFMA)
    pme.set_gemm_tile(tile)
    y = pme.fp8_gemm(*ops[:4])
    torch.cuda.synchronize()
    check_gemm(y, ops[:4])
    if tile > 202:                                    # tiles of 16 rows of weights have no room for two matrices
        z = pme.fp8_gated_gemm(*ops)
        torch.cuda.synchronize()
        check_gated(z, ops)


@pytest.mark.parametrize("T,K,N,first,gated", [(905, 768, 4141, 4096, True), (2845, 768, 2817, 2816, False), (226, 2048, 8444, 8192, True)])
def test_whole_rounds_and_the_channels_behind_them(T, K, N, first, gated):
    """Shapes whose last channels another tile computes: the first block of 128 channels, the last one before them, and themselves."""
    ops = _operands(T, K, N, T + N, mats=2 if gated else 1)
    y = (pme.fp8_gated_gemm if gated else pme.fp8_gemm)(*ops)
    torch.cuda.synchronize()
    assert not bool(torch.isnan(y).any())
    blocks = [0, first // 128 - 1, *range(first // 128, (N + 127) // 128)]
    rows = torch.cat([torch.arange(128 * b, min(128 * b + 128, N)) for b in blocks]).cuda()
    part = ops[:2]
    for q, s in zip(ops[2::2], ops[3::2]):
        part += [q.view(torch.uint8)[rows].view(torch.float8_e4m3fn), s[torch.tensor(blocks).cuda()]]
    (check_gated if gated else check_gemm)(y[:, rows], part)


def test_operands_beyond_4_gib():
    """Codes of more than 2^32 bytes, as tokens and as weights: rows on both sides of the place where a launch's offsets end, and the last one."""
    K, rows = 14336, 300032
    cut = ((1 << 32) - 1) // K // 256 * 256
    gen = torch.Generator(device="cuda")
    gen.manual_seed(7)
    big = torch.randint(0, 0x78, (rows, K), dtype=torch.uint8, device="cuda", generator=gen)
    big[:, ::2] |= 0x80
    big = big.view(torch.float8_e4m3fn)
    sx = torch.rand((rows, K // 128), device="cuda", generator=gen) * 1e-3
    sw = torch.rand(((rows + 127) // 128, K // 128), device="cuda", generator=gen) * 1e-3
    qs, ss = _operands(40, K, 72, 11)[2:]                                         # 72 channels
    qt, st = _operands(5, K, 8, 12)[:2]                                           # 5 tokens
    at = torch.tensor([0, 127, cut - 1, cut, cut + 130, rows - 1], device="cuda")
    pick = big.view(torch.uint8)[at].view(torch.float8_e4m3fn)
    y = pme.fp8_gemm(big, sx, qs, ss)
    torch.cuda.synchronize()
    check_gemm(y[at], [pick, sx[at], qs, ss])
    y = pme.fp8_gemm(qt, st, big, sw)
    z = pme.fp8_gated_gemm(qt, st, big, sw, big, sw)
    torch.cuda.synchronize()
    for i, row in enumerate(at.tolist()):
        one = [pick[i:i + 1], sw[row // 128:row // 128 + 1]]
        check_gemm(y[:, row:row + 1], [qt, st, *one])
        check_gated(z[:, row:row + 1], [qt, st, *one, *one])


def test_products_write_their_columns_only():
    for T, K, N in ((5, 256, 67), (150, 512, 333)):
        ops = _operands(T, K, N, 9, mats=2)
        for f, o in ((pme.fp8_gemm, ops[:4]), (pme.fp8_gated_gemm, ops)):
            whole = f(*o)
            for pad, first in ((13, 0), (16, 8), (7, 3)):
                big = torch.full((T + 3, N + pad), 7.0, dtype=torch.bfloat16, device="cuda")
                f(*o, big[:T, first:first + N])
                torch.cuda.synchronize()
                assert torch.equal(big[:T, first:first + N], whole)
                assert bool((big[T:] == 7).all()) and bool((big[:T, :first] == 7).all()) and bool((big[:T, first + N:] == 7).all())


def test_nan_codes_reach_their_rows_only():
    ops = _operands(40, 384, 200, 3)
    clean = pme.fp8_gemm(*ops)
    ops[1][7, 1] = float("nan")                       # as the quantizers mark a block that is not finite
    y = pme.fp8_gemm(*ops)
    torch.cuda.synchronize()
    assert bool(torch.isnan(y[7]).all())
    assert torch.equal(y[:7], clean[:7]) and torch.equal(y[8:], clean[8:])


@pytest.mark.parametrize("tile", TILES)
def test_scales_that_are_not_finite_reach_their_rows_and_channels_only(tile):
    """Blocks of K that fill no group of four scales and no whole step of the slices of K: the scales that follow a row's in memory are its neighbour's."""
    for K in (128, 256, 384, 640, 1152, 1408):
        ops = _operands(72, K, 300, 5, mats=2)
        pme.set_path(pme.PATH_MFMA)
        pme.set_gemm_tile(tile)
        for f, o in ((pme.fp8_gemm, ops[:4]), (pme.fp8_gated_gemm, ops)):
            if tile < 203 and f is pme.fp8_gated_gemm:
                continue
            clean = f(*o)
            sx, sw = ops[1].clone(), ops[3].clone()
            sx[7, 0], sx[40, -1], sx[41], sx[71, 0] = float("nan"), float("inf"), float("nan"), float("nan")
            sw[1, 0] = float("nan")
            y = f(o[0], sx, o[2], sw, *o[4:])
            torch.cuda.synchronize()
            bad = torch.zeros_like(y, dtype=torch.bool)
            bad[[7, 41, 71]] = True
            bad[:, 128:256] = True
            assert bool(torch.isnan(y[bad]).all())
            bad[40] = True                                # infinite, or NaN where infinities cancel
            assert torch.equal(y[~bad], clean[~bad])


@pytest.mark.parametrize("tile", [0, *TILES])
def test_products_of_scales_over_fp32s_normal_range(tile):
    """Powers of two, whose products are the smallest and the largest normal ones and some between: exact but for the sum's one bf16 rounding."""
    x, w = torch.zeros((8, 256), device="cuda"), torch.zeros((24, 256), device="cuda")
    x[:, 3], x[:, 130], w[:, 3], w[:, 130] = 1.0, 0.5, 0.25, 1.0      # 1/4 + 1/2 of the product of the scales
    x, w = x.to(torch.float8_e4m3fn), w.to(torch.float8_e4m3fn)
    pme.set_path(pme.PATH_MFMA if tile else pme.PATH_GENERIC)
    pme.set_gemm_tile(tile)
    for total in (-126, -20, 0, 90, 127):
        for t in (-126, -100, -63, -1, 0, 30, 64, 127):
            if not -126 <= total - t <= 127:
                continue
            sx = torch.full((8, 2), 2.0 ** t, device="cuda")
            sw = torch.full((1, 2), 2.0 ** (total - t), device="cuda")
            y = pme.fp8_gemm(x, sx, w, sw)
            torch.cuda.synchronize()
            assert bool((y.double() == 0.75 * 2.0 ** total).all()), (total, t)


def test_gate_over_its_range():
    """g = u = the token's scale: half a step of bf16, eight of fp32's roundings, and what a reciprocal below 2^-126 may lose."""
    g = torch.cat([torch.linspace(-130.0, 130.0, 2601), torch.tensor([0.0, 1e-30, -1e-30, 1e15, -1e15, -87.3, -88.0, -88.8])]).cuda()[:, None]
    x = torch.zeros((len(g), 128), device="cuda")
    x[:, 5] = 1.0
    x, w, one = x.to(torch.float8_e4m3fn), x[:300].to(torch.float8_e4m3fn), torch.ones((3, 1), device="cuda")
    v = _f64(g)
    with np.errstate(over="ignore"):
        ref = v / (1 + np.exp(-v)) * v
    for tile in (0, 203, 204, 205, 206, 207, 208, 209, 210, 211, 212, 213):
        pme.set_gemm_tile(tile)
        y = pme.fp8_gated_gemm(x, g, w, one, w, one)
        torch.cuda.synchronize()
        # bf16's numbers are 2^-133 apart below 2^-126: half of that is lost where 1e-30 comes out as 5e-61, which no bf16 is near
        lim = (2.0 ** -8 + 8 * U) * np.abs(ref) + 2.0 ** -119 * np.abs(v) + 2.0 ** -134
        err = np.abs(_f64(y) - ref)
        assert np.all(err <= lim), (tile, v[(err > lim).any(axis=1)][:9, 0])
    y = pme.fp8_gated_gemm(x[:1], torch.full((1, 1), float("nan"), device="cuda"), w, one, w, one)
    torch.cuda.synchronize()
    assert bool(torch.isnan(y).all())


@pytest.mark.parametrize("tile", [0, *TILES])
def test_rows_and_blocks_of_channels_of_larger_operands(tile):
    """Views of tokens and of blocks of channels: scales aligned to 4 bytes only where a row has an odd number of them, codes to 16 and more."""
    ops = _operands(70, 640, 400, 21, mats=2)
    view = [ops[0][3:], ops[1][3:], ops[2][128:], ops[3][1:], ops[4][128:], ops[5][1:]]
    pme.set_path(pme.PATH_MFMA)
    pme.set_gemm_tile(tile)
    y = pme.fp8_gemm(*view[:4])
    torch.cuda.synchronize()
    check_gemm(y, view[:4])
    if tile not in (201, 202):
        z = pme.fp8_gated_gemm(*view)
        torch.cuda.synchronize()
        check_gated(z, view)


# ---- together

def _block(seed, T=70, d=640, f=704, f_e=768):
    """A feed-forward block: norm, gated product, expanded int4 down projection."""
    wg, wu = _rand((f, d), seed, outliers=False) / d ** 0.5, _rand((f, d), seed + 1, outliers=False) / d ** 0.5
    wd = _rand((d, f), seed + 2, outliers=False) / f ** 0.5
    return {"x": _rand((T, d), seed + 3), "r": _rand((T, d), seed + 4), "w": _rand((1, d), seed + 5, outliers=False)[0], "d_e": f_e,
            "g": pme.quantize_weights_fp8(wg), "u": pme.quantize_weights_fp8(wu), "down": pme.expand_quantize_weights(wd, f_e)}


def _run_block(b, r):
    q, s, h = pme.rmsnorm_quant_fp8(b["x"], b["w"], EPS, r)
    a = pme.fp8_gated_gemm(q, s, *b["g"], *b["u"])
    return pme.expanded_linear(a, b["d_e"], *b["down"]), h, a, q, s


def test_feed_forward_block():
    b = _block(50)
    y, h, a, q, s = _run_block(b, b["r"])
    torch.cuda.synchronize()
    assert torch.equal(h, (b["x"].float() + b["r"].float()).to(torch.bfloat16))
    check_codes(q, s, *oracle.fp8_quotients(oracle.rmsnorm(_f64(h), _f64(b["w"]), EPS)), norm_delta(h.shape[1]))
    check_gated(a, [q, s, *b["g"], *b["u"]])
    ref = oracle.expanded_linear(_f64(a), b["d_e"], oracle.unpack_int4(b["down"][0].cpu().numpy()), b["down"][1].cpu().numpy())
    # codes of the down projection that sit at a tie may differ: a flip moves an output by a weight code (at most 8) times both scales
    step = 8 * ref["sx"][:, None] * b["down"][1].cpu().numpy()[None]
    assert np.all(np.abs(_f64(y) - ref["y"]) <= 1e-2 * np.abs(ref["y"]) + 2 * step)


def test_block_on_another_stream_and_replayed():
    """The block captured into a graph: every replay, with the program's own work between, equals the eager run on the same inputs."""
    b = _block(80, T=33)
    want = [t.clone() for t in _run_block(b, b["r"])]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _run_block(b, b["r"])
    side.synchronize()
    assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    r = b["r"].clone()
    with torch.cuda.graph(graph):
        out = _run_block(b, r)
    for k in range(4):
        r.copy_(b["r"] * (k + 1))
        graph.replay()
        torch.cuda.synchronize()
        eager = _run_block(b, b["r"] * (k + 1))
        torch.cuda.synchronize()
        assert all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(eager, out))


# ---- more rows than a grid has workgroups for: each takes further ones

@pytest.mark.parametrize("xt", ["bf16", "f32"])
def test_quant_rows_beyond_the_grid(xt):
    cap, T, d = 1 << 15, (1 << 16) + 70, 130
    x = torch.randn((T, d), device="cuda", generator=torch.Generator("cuda").manual_seed(1)).to(DT[xt])
    q, s = pme.quant_fp8(x)
    parts = [pme.quant_fp8(x[i:i + cap]) for i in range(0, T, cap)]
    torch.cuda.synchronize()
    assert torch.equal(q.view(torch.uint8), torch.cat([p[0].view(torch.uint8) for p in parts])) and torch.equal(s, torch.cat([p[1] for p in parts]))
    at = [0, cap - 1, cap, cap + 1, 2 * cap, T - 1]
    check_codes(q.view(torch.uint8)[at].view(q.dtype), s[at], *oracle.fp8_quotients(_f64(x[at])), 0.0)


# a wave, several waves with one chunk a lane, and with two, for a row
@pytest.mark.parametrize("cap,d,residual", [(1 << 22, 8, True), (1 << 20, 520, True), (1 << 20, 1544, False)])
def test_rmsnorm_rows_beyond_the_grid(cap, d, residual):
    T, gen = cap + 3000, torch.Generator("cuda").manual_seed(2)      # (the rows behind go by themselves on the same kernel)
    x = torch.randn((T, d), device="cuda", generator=gen, dtype=torch.bfloat16)
    r = torch.randn((T, d), device="cuda", generator=gen, dtype=torch.bfloat16) if residual else None
    x[cap + 2000] *= 1e30                             # squares that overflow: the row's further sums, on the other of its two places
    w = torch.randn((d,), device="cuda", generator=gen)
    whole = pme.rmsnorm_quant_fp8(x, w, EPS, r)
    parts = [pme.rmsnorm_quant_fp8(x[i:j], w, EPS, r[i:j] if residual else None) for i, j in ((0, cap), (cap, T))]
    torch.cuda.synchronize()
    for got, *want in zip(whole, *parts):
        got, want = got.view(torch.uint8), torch.cat([t.view(torch.uint8) for t in want])
        assert torch.equal(got, want)
    at = [0, cap - 1, cap, cap + 1, cap + 2000, T - 1]
    h = (x[at].float() + r[at].float()).to(torch.bfloat16) if residual else x[at]
    if residual:
        assert torch.equal(whole[2][at], h)
    check_codes(whole[0].view(torch.uint8)[at].view(whole[0].dtype), whole[1][at], *oracle.fp8_quotients(oracle.rmsnorm(_f64(h), _f64(w), EPS)), norm_delta(d) + 4 * U)


def test_weight_blocks_beyond_the_grid():
    cap, d = 128 << 15, 130
    N = cap + 300
    w = torch.randn((N, d), device="cuda", generator=torch.Generator("cuda").manual_seed(3), dtype=torch.bfloat16)
    w[cap - 128:cap] *= 100.0                         # neighbouring blocks of other scales
    w[cap + 128:cap + 256] *= 0.01
    q, s = pme.quantize_weights_fp8(w)
    parts = [pme.quantize_weights_fp8(w[:cap]), pme.quantize_weights_fp8(w[cap:])]
    torch.cuda.synchronize()
    assert torch.equal(q.view(torch.uint8), torch.cat([p[0].view(torch.uint8) for p in parts])) and torch.equal(s, torch.cat([p[1] for p in parts]))
    check_codes(q[cap - 128:], s[(cap - 128) // 128:], *oracle.fp8_quotients_weights(_f64(w[cap - 128:])), 0.0)


_COLD_SCRIPT = """
import sys, torch
sys.path.insert(0, sys.argv[1])
import paper_2503_17513_amd as pme
FP8, gen = torch.float8_e4m3fn, torch.Generator("cuda").manual_seed(5)
def codes(rows, K):
    return (torch.randn((rows, K), device="cuda", generator=gen) * 100).clamp(-448, 448).to(FP8)
def scales(rows, K):
    return torch.rand((rows, K // 128), device="cuda", generator=gen) * 1e-3
T, K, N = 70, 640, 300
x, r, w = torch.randn((T, 600), device="cuda", generator=gen), torch.randn((T, 600), device="cuda", generator=gen), torch.ones(600, device="cuda")
wide = torch.randn((3, 40000), device="cuda", generator=gen).to(torch.bfloat16)
wide_w = torch.ones(40000, device="cuda", dtype=torch.bfloat16)
ops = [codes(T, K), scales(T, K)] + [f(n, K) for _ in range(2) for f, n in ((codes, N), (scales, 3))]
calls = [lambda: pme.rmsnorm_quant_fp8(x, w, 1e-5, r), lambda: pme.rmsnorm_quant_fp8(wide, wide_w, 1e-5), lambda: pme.quant_fp8(x),
         lambda: pme.quant_fp8(wide), lambda: pme.quantize_weights_fp8(x), lambda: pme.quantize_weights_fp8(wide)]
def product(f, o, path, tile):
    def call():
        pme.set_path(path)
        pme.set_gemm_tile(tile)
        y = f(*o)
        pme.set_gemm_tile(0)
        pme.set_path(pme.PATH_AUTO)
        return [y]
    return call
for f, o in ((pme.fp8_gemm, ops[:4]), (pme.fp8_gated_gemm, ops)):
    calls.append(product(f, o, pme.PATH_GENERIC, 0))
    calls.append(product(f, o, pme.PATH_AUTO, 0))
    for tile in range(201 if f is pme.fp8_gemm else 203, 214):
        calls.append(product(f, o, pme.PATH_MFMA, tile))
torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph, stream=torch.cuda.Stream()):      # the process's first call of every one of them
    out = [[t.view(torch.uint8) for t in call()] for call in calls]
for _ in range(3):
    for ts in out:
        for t in ts:
            t.fill_(0xA5)
    torch.cuda.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    got = [[t.clone() for t in ts] for ts in out]
    want = [[t.view(torch.uint8) for t in call()] for call in calls]
    torch.cuda.synchronize()
    for i, (a, b) in enumerate(zip(got, want)):
        assert all(torch.equal(p, q) for p, q in zip(a, b)), i
print("COLD_OK", len(calls))
"""


def test_first_calls_of_all_kernels_are_captured():
    # in a process of its own: here every kernel has run
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    p = subprocess.run([sys.executable, "-c", _COLD_SCRIPT, root], capture_output=True, text=True, timeout=110)
    assert p.returncode == 0 and "COLD_OK 34" in p.stdout, p.stdout[-2000:] + p.stderr[-2000:]


# tokens, features, channels, first channel of the second kernel, gated, the first kernel and the tile that forces it
@pytest.mark.parametrize("T,K,N,first,gated,kernel,tile,second", [
    (396, 2048, 4142, 4096, True, "k_fp8_gemm<128, 128, 4, 2, ", 210, "k_fp8_gemm_kslice<8, 32, "), (641, 2048, 5432, 5376, False, "k_fp8_gemm<128, 128, 4, 2, ", 210, "k_fp8_gemm_kslice<16, 16, "),
    (670, 1024, 5445, 5376, True, "k_fp8_gemm<128, 256, ", 212, "k_fp8_gemm_kslice<16, 32, "), (1288, 1024, 5908, 5888, False, "k_fp8_gemm<128, 256, ", 212, "k_fp8_gemm_kslice<16, 16, "),
    (913, 1024, 11597, 8192, True, "k_fp8_gemm<256, 256, ", 213, "k_fp8_gemm<128, 256, "), (1426, 1152, 11767, 10752, False, "k_fp8_gemm<256, 256, ", 213, "k_fp8_gemm<64, 128, ")])
def test_whole_rounds_on_one_kernel_and_the_rest_on_another(T, K, N, first, gated, kernel, tile, second):
    """That two kernels run, where they meet, and both: the channels of the first as from it alone, some blocks of both against the oracle."""
    assert pme.fp8_gemm_plan(T, K, N, gated=gated).startswith(kernel)
    rest = pme.fp8_gemm_rest(T, K, N, gated=gated)
    assert rest[0] == first and rest[1].startswith(second)
    ops = _operands(T, K, N, T + N, mats=2 if gated else 1)
    f = pme.fp8_gated_gemm if gated else pme.fp8_gemm
    big = torch.full((T + 1, N + 3), float("nan"), dtype=torch.bfloat16, device="cuda")
    y = f(*ops, big[:T, 1:1 + N])
    pme.set_gemm_tile(tile)
    assert pme.fp8_gemm_rest(T, K, N, gated=gated) == (N, "")
    alone = f(*ops)
    torch.cuda.synchronize()
    assert not bool(torch.isnan(y).any()) and bool(torch.isnan(big[T]).all()) and bool(torch.isnan(big[:, [0, N + 1, N + 2]]).all())
    assert torch.equal(y[:, :first], alone[:, :first])
    tokens = torch.tensor(sorted({*range(16), *range(0, T, 9), *range(T - 16, T)})).cuda()
    blocks = sorted({0, first // 128 - 1, first // 128, first // 128 + 1, (N - 1) // 128} & set(range((N + 127) // 128)))
    rows = torch.cat([torch.arange(128 * b, min(128 * b + 128, N)) for b in blocks]).cuda()
    part = [ops[0].view(torch.uint8)[tokens].view(torch.float8_e4m3fn), ops[1][tokens]]
    for q, s in zip(ops[2::2], ops[3::2]):
        part += [q.view(torch.uint8)[rows].view(torch.float8_e4m3fn), s[torch.tensor(blocks).cuda()]]
    (check_gated if gated else check_gemm)(y[tokens][:, rows], part)
