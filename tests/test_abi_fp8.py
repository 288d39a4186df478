"""Host-side tests of the 8-bit entry points: every refusal, before any HIP call, and what the binding refuses."""
import ctypes as C

import pytest
import torch

import paper_2503_17513_amd as pme
from test_abi_host import _kernel_metadata

OK, NULL, SHAPE, ORDER, ALIGN, WORKSPACE, DTYPE, HIP, PATH, COLD = range(10)
FAKE = 0x10000   # a non-null, 64 KiB aligned address that is never dereferenced: every call below fails validation
NAN, INF = float("nan"), float("inf")


def test_rmsnorm_quant_fp8_argument_errors():
    f = pme.lib().pme_rmsnorm_quant_fp8

    def call(x=FAKE, xt=1, T=4, d=130, ldx=130, r=FAKE, ldr=130, h=FAKE, ldh=130, w=FAKE, wt=1, eps=1e-5, q=FAKE, s=FAKE):
        return f(x, xt, T, d, ldx, r, ldr, h, ldh, w, wt, eps, q, s, None)

    assert call(x=None) == call(w=None) == call(q=None) == call(s=None) == NULL
    assert call(r=None) == call(h=None) == NULL                      # both or neither
    assert call(xt=2) == call(wt=7) == DTYPE
    assert call(T=-1) == call(d=0) == call(d=-5) == call(ldx=129) == call(ldr=129) == call(ldh=129) == SHAPE
    assert call(T=1 << 31) == call(d=(1 << 20) + 1, ldx=1 << 21, ldr=1 << 21, ldh=1 << 21) == SHAPE
    assert call(eps=-1e-9) == call(eps=NAN) == call(eps=INF) == SHAPE
    assert call(x=FAKE + 1) == call(xt=0, x=FAKE + 2) == call(r=FAKE + 1) == call(h=FAKE + 1) == call(w=FAKE + 1) == call(wt=0, w=FAKE + 2) == ALIGN
    assert call(q=FAKE + 8) == call(s=FAKE + 2) == ALIGN
    assert call(T=0, x=None, r=None, h=None, w=None, q=None, s=None) == OK


def test_quantizers_argument_errors():
    for f in (pme.lib().pme_quant_fp8, pme.lib().pme_quantize_weights_fp8):
        def call(x=FAKE, xt=1, T=4, d=130, ldx=130, q=FAKE, s=FAKE):
            return f(x, xt, T, d, ldx, q, s, None)

        assert call(x=None) == call(q=None) == call(s=None) == NULL
        assert call(xt=-1) == DTYPE
        assert call(T=-1) == call(d=0) == call(ldx=129) == call(T=1 << 31) == call(d=(1 << 20) + 1, ldx=1 << 21) == SHAPE
        assert call(x=FAKE + 1) == call(xt=0, x=FAKE + 2) == call(q=FAKE + 4) == call(s=FAKE + 1) == ALIGN
        assert call(T=0, x=None, q=None, s=None) == OK


def test_fp8_gemm_argument_errors():
    f = pme.lib().pme_fp8_gemm

    def call(qx=FAKE, sx=FAKE, qw=FAKE, sw=FAKE, T=4, K=256, N=8, y=FAKE, ldy=8):
        return f(qx, sx, qw, sw, T, K, N, y, ldy, None)

    assert call(qx=None) == call(sx=None) == call(qw=None) == call(sw=None) == call(y=None) == NULL
    assert call(T=-1) == call(N=-1) == call(K=0) == call(K=64) == call(K=200) == call(ldy=7) == SHAPE
    assert call(T=1 << 31) == call(N=1 << 31, ldy=1 << 31) == call(K=(1 << 20) + 128) == SHAPE
    assert call(qx=FAKE + 8) == call(qw=FAKE + 4) == call(sx=FAKE + 2) == call(sw=FAKE + 1) == call(y=FAKE + 1) == ALIGN
    assert call(T=0, qx=None) == call(N=0, ldy=0) == OK


def test_fp8_gated_gemm_argument_errors():
    f = pme.lib().pme_fp8_gated_gemm

    def call(qx=FAKE, sx=FAKE, qg=FAKE, sg=FAKE, qu=FAKE, su=FAKE, T=4, K=256, N=8, y=FAKE, ldy=8):
        return f(qx, sx, qg, sg, qu, su, T, K, N, y, ldy, None)

    assert call(qx=None) == call(sx=None) == call(qg=None) == call(sg=None) == call(qu=None) == call(su=None) == call(y=None) == NULL
    assert call(T=-1) == call(K=130) == call(ldy=7) == SHAPE
    assert call(qu=FAKE + 8) == call(su=FAKE + 2) == call(qg=FAKE + 8) == call(y=FAKE + 1) == ALIGN
    assert call(T=0, qu=None) == call(N=0, ldy=0) == OK


def test_fp8_gemm_plan_argument_errors():
    f, buf = pme.lib().pme_fp8_gemm_plan, C.create_string_buffer(64)
    assert f(0, 4, 256, 8, None, 64) == f(0, 4, 256, 8, buf, 0) == NULL
    assert f(0, 0, 256, 8, buf, 64) == f(1, 4, 256, 0, buf, 64) == f(0, 4, 200, 8, buf, 64) == SHAPE
    assert f(1, 4, 256, 8, buf, 64) == OK and buf.value.startswith(b"k_fp8_")


def test_fp8_gemm_rest():
    f, buf, first = pme.lib().pme_fp8_gemm_rest, C.create_string_buffer(64), C.c_int64(-5)
    at = C.byref(first)
    assert f(0, 4, 256, 8, None, buf, 64) == f(0, 4, 256, 8, at, None, 64) == f(0, 4, 256, 8, at, buf, 0) == NULL
    assert f(0, 0, 256, 8, at, buf, 64) == f(1, 4, 256, 0, at, buf, 64) == f(0, 4, 200, 8, at, buf, 64) == SHAPE
    assert first.value == -5                                          # untouched where the call is refused
    assert f(0, 4, 256, 8, at, buf, 64) == OK and first.value == 8 and buf.value == b""
    first, name = pme.fp8_gemm_rest(1999, 4096, 14336, gated=True)    # 3.5 rounds of 256 x 256
    assert first == 12288 and name.startswith("k_fp8_gemm<128, 256, ")
    try:
        pme.set_path(pme.PATH_GENERIC)
        assert pme.fp8_gemm_rest(1999, 4096, 14336, gated=True) == (14336, "")
        pme.set_path(pme.PATH_AUTO)
        pme.set_gemm_tile(213)                                        # a forced tile computes everything
        assert pme.fp8_gemm_rest(1999, 4096, 14336, gated=True) == (14336, "")
    finally:
        pme.set_gemm_tile(0)
        pme.set_path(pme.PATH_AUTO)


# tokens, features, channels, gated, the tile estimated fastest
@pytest.mark.parametrize("T,K,N,gated,kernel", [
    (1, 8192, 2048, False, "k_fp8_gemm_kslice<8, 16, "), (16, 14336, 4096, False, "k_fp8_gemm_kslice<16, 16, "), (8, 2048, 8192, True, "k_fp8_gemm_kslice<16, 32, "), (2, 4096, 2048, True, "k_fp8_gemm_kslice<8, 32, "),
    (16, 4096, 14336, True, "k_fp8_gemm_kslice<16, 32, "), (64, 4096, 4096, False, "k_fp8_gemm_kslice<32, 32, "), (128, 4096, 4096, False, "k_fp8_gemm_kslice<64, 32, "),
    (333, 4096, 4096, False, "k_fp8_gemm<64, 128, "), (517, 4096, 4096, False, "k_fp8_gemm<128, 128, "), (2048, 4096, 4096, False, "k_fp8_gemm<128, 256, "),
    (4096, 14336, 4096, False, "k_fp8_gemm<256, 256, "), (1999, 4096, 14336, True, "k_fp8_gemm<256, 256, ")])
def test_fp8_gemm_plan_by_fitted_times(T, K, N, gated, kernel):
    assert pme.fp8_gemm_plan(T, K, N, gated=gated).startswith(kernel)


# operands beyond 4 GiB go in slices of 299520 rows of 14336 codes, or of 3840 rows of 2^20
@pytest.mark.parametrize("T,K,N,first,gated", [(300032, 14336, 72, (299520, 14336, 72), False), (200, 14336, 300032, (200, 14336, 299520), True),
                                               (1 << 24, 1 << 20, 1 << 20, (3840, 1 << 20, 3840), False)])
def test_fp8_gemm_plan_names_the_kernel_of_the_first_slice(T, K, N, first, gated):
    assert pme.fp8_gemm_plan(T, K, N, gated=gated) == pme.fp8_gemm_plan(*first, gated=gated)
    assert pme.fp8_gemm_plan(T, K, N, gated=gated) != pme.fp8_gemm_plan(T % first[0] or T, K, N % first[2] or N, gated=gated)


def test_a_forced_fp8_tile_that_refuses_is_not_replaced():
    f, buf = pme.lib().pme_fp8_gemm_plan, C.create_string_buffer(96)
    try:
        for tile, gated in ((201, 1), (202, 1), (214, 0), (299, 1)):
            pme.set_gemm_tile(tile)
            assert pme.fp8_gemm_plan(8, 512, 300, gated=bool(gated)).startswith("k_fp8_gemm_generic<")
            pme.set_path(pme.PATH_MFMA)
            assert f(gated, 8, 512, 300, buf, 96) == PATH
            pme.set_path(pme.PATH_AUTO)
        pme.set_gemm_tile(201)
        assert pme.fp8_gemm_plan(8, 512, 300) == "k_fp8_gemm_kslice<8, 16, 4, 5, false>"
    finally:
        pme.set_gemm_tile(0)
        pme.set_path(pme.PATH_AUTO)


def test_fp8_kernels_use_no_scratch():
    # accumulators, fragments and rows stay in registers
    kernels = [k for k in _kernel_metadata() if any(n in k[".name"] for n in ("k_fp8_gemm", "_quant_fp8", "k_quantize_weights_fp8", "Fp8TileArgs", "NormQuantArgs"))]
    assert len(kernels) >= 2 * 13 - 2 + 2 + 2 * 2 + 8 * 5
    assert not [k[".name"] for k in kernels if k[".private_segment_fixed_size"] or k[".vgpr_spill_count"]]


def test_binding_refuses_host_tensors_and_wrong_operands():
    x, w = torch.zeros(2, 130), torch.zeros(130)
    with pytest.raises(ValueError):
        pme.rmsnorm_quant_fp8(x, w, 1e-5)
    with pytest.raises(ValueError):
        pme.quant_fp8(x)
    with pytest.raises(ValueError):
        pme.quantize_weights_fp8(x)
    with pytest.raises(TypeError):
        pme.quant_fp8(x.to(torch.float16))
    with pytest.raises(ValueError):
        pme.rmsnorm_quant_fp8(x, w[:5], 1e-5)                         # weight of another width
    with pytest.raises(ValueError):
        pme.rmsnorm_quant_fp8(x, w, 1e-5, h=x)                        # a sum without a residual
    with pytest.raises(ValueError):
        pme.rmsnorm_quant_fp8(x, w, 1e-5, residual=x.to(torch.bfloat16))
    with pytest.raises(ValueError):
        pme.quant_fp8(x, qx=torch.zeros((2, 130), dtype=torch.float8_e4m3fn))      # rows are whole groups
    with pytest.raises(ValueError):
        pme.quant_fp8(x, sx=torch.zeros((2, 1)))
    q, s = torch.zeros((2, 256), dtype=torch.float8_e4m3fn), torch.zeros((2, 2))
    qw, sw = torch.zeros((130, 256), dtype=torch.float8_e4m3fn), torch.zeros((2, 2))
    with pytest.raises(ValueError):
        pme.fp8_gemm(q, s, qw, sw)                                    # host tensors
    with pytest.raises(ValueError):
        pme.fp8_gemm(q.view(torch.uint8), s, qw, sw)
    with pytest.raises(ValueError):
        pme.fp8_gemm(q, s[:1], qw, sw)
    with pytest.raises(ValueError):
        pme.fp8_gemm(q, s, qw, sw[:1])                                # a scale for each 128 channels
    with pytest.raises(ValueError):
        pme.fp8_gemm(q[:, :128].contiguous(), s[:, :1].contiguous(), qw, sw)
    with pytest.raises(ValueError):
        pme.fp8_gated_gemm(q, s, qw, sw, qw[:129].contiguous(), sw)
    with pytest.raises(ValueError):
        pme.fp8_gemm(q, s, qw, sw, torch.zeros((2, 130)))             # y in another type
