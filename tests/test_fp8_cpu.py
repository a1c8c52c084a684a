"""The 8-bit matrices of include/sbw_step.h on the CPU: bad arguments are refused before any HIP call, by the
C entry points and by the Python ones; the reference's own rounding."""
import ctypes

import numpy as np
import pytest
import torch

import fp8_reference as ref

OK, INVALID, GAMMA, DELTA, UNSUPPORTED, NO_DEVICE, HIP = range(7)
DUMMY = ctypes.c_void_p(0x1000)   # rejected before it could be used
E8M0 = torch.float8_e8m0fnu


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


@pytest.fixture(scope="module")
def lib(sbw):
    return sbw.raw()


def quantize(lib, x=DUMMY, dtype=0, M=4, K=200, stride=200, rows=1, kind=0, codes=DUMMY, cs=200, scales=DUMMY,
             codes_t=None, cts=4, scales_t=None):
    return lib.sbw_quantize_fp8(x, dtype, M, K, stride, rows, kind, codes, cs, scales, codes_t, cts, scales_t, None)


def test_quantize_refusals(lib):
    assert quantize(lib, M=-1) == INVALID
    assert quantize(lib, K=-1) == INVALID
    assert quantize(lib, stride=199) == INVALID
    assert quantize(lib, cs=199) == INVALID
    assert quantize(lib, codes_t=DUMMY, scales_t=DUMMY, cts=3) == INVALID
    assert quantize(lib, x=None) == INVALID
    assert quantize(lib, codes=None) == INVALID                    # scales without codes
    assert quantize(lib, scales=None) == INVALID
    assert quantize(lib, codes_t=DUMMY) == INVALID
    assert quantize(lib, codes=None, scales=None) == INVALID       # nothing to write
    for rows in (0, 2, 64, -1, 256):
        assert quantize(lib, rows=rows) == UNSUPPORTED
    assert quantize(lib, dtype=2) == UNSUPPORTED
    assert quantize(lib, kind=2) == UNSUPPORTED
    assert quantize(lib, M=1 << 31) == UNSUPPORTED
    assert quantize(lib, K=1 << 31, stride=1 << 31, cs=1 << 31) == UNSUPPORTED
    assert quantize(lib, stride=1 << 62) == UNSUPPORTED
    assert quantize(lib, M=0, x=None) == OK
    assert quantize(lib, K=0, x=None) == OK


def product(lib, a=DUMMY, M=4, a_stride=256, sa=DUMMY, ra=1, b=DUMMY, N=8, b_stride=256, sb=DUMMY, rb=128, K=256, kind=0,
            out=DUMMY, dtype=0, stride=8, ws=DUMMY):
    return lib.sbw_matmul_fp8(a, M, a_stride, sa, ra, b, N, b_stride, sb, rb, K, kind, out, dtype, stride, ws, None)


def test_matmul_refusals(lib):
    assert product(lib, M=-1) == INVALID
    assert product(lib, N=-1) == INVALID
    assert product(lib, K=0) == INVALID
    assert product(lib, K=-5) == INVALID
    assert product(lib, a_stride=255) == INVALID
    assert product(lib, b_stride=255) == INVALID
    assert product(lib, stride=7) == INVALID
    for name in ("a", "b", "sa", "sb", "out"):
        assert product(lib, **{name: None}) == INVALID, name
    for rows in (0, 2, 127):
        assert product(lib, ra=rows) == UNSUPPORTED
        assert product(lib, rb=rows) == UNSUPPORTED
    assert product(lib, dtype=2) == UNSUPPORTED
    assert product(lib, kind=-1) == UNSUPPORTED
    assert product(lib, a_stride=1 << 23) == UNSUPPORTED
    assert product(lib, b_stride=1 << 23) == UNSUPPORTED
    assert product(lib, M=1 << 23) == UNSUPPORTED
    assert product(lib, N=1 << 30, stride=1 << 30) == UNSUPPORTED
    assert product(lib, stride=1 << 62) == UNSUPPORTED
    assert product(lib, M=1 << 20, N=1 << 20, stride=1 << 20) == UNSUPPORTED      # more tiles than a launch takes
    assert product(lib, M=0) == OK
    assert product(lib, N=0, stride=0) == OK
    for sizes in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (-1, 5, 5), (1 << 40, 5, 5)):
        assert lib.sbw_matmul_fp8_workspace(*sizes) == 0
    if lib.sbw_matmul_fp8_workspace(64, 64, 16384) > 0:
        assert product(lib, M=64, N=64, K=16384, a_stride=16384, b_stride=16384, stride=64, ws=None) == INVALID


def codes(M, K, device="cpu"):
    return torch.zeros((M, K), dtype=torch.uint8, device=device).view(torch.float8_e4m3fn)


def scales(M, K, dtype=E8M0):
    return torch.ones((M, K)).to(dtype)


def test_python_refusals_of_quantize(sbw):
    x = torch.zeros((4, 300))
    with pytest.raises(ValueError, match="current HIP device"):
        sbw.quantize_fp8(x)
    with pytest.raises(TypeError):
        sbw.quantize_fp8(x.half())
    with pytest.raises(TypeError):
        sbw.quantize_fp8(x, scale_dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="two-dimensional"):
        sbw.quantize_fp8(x[0])
    with pytest.raises(ValueError, match="unit stride"):
        sbw.quantize_fp8(x.t())
    with pytest.raises(ValueError, match="overlap"):
        sbw.quantize_fp8(x[:1].expand(3, 300))
    with pytest.raises(ValueError, match="no gradient"):
        sbw.quantize_fp8(x.clone().requires_grad_())
    with pytest.raises(ValueError, match="negated"):
        sbw.quantize_fp8(torch._neg_view(x))
    with pytest.raises(ValueError, match="codes must be"):
        sbw.quantize_fp8(x, codes=codes(4, 299))
    with pytest.raises(ValueError, match="float8_e4m3fn"):
        sbw.quantize_fp8(x, codes=torch.zeros((4, 300), dtype=torch.uint8))
    with pytest.raises(ValueError, match="scales must be"):
        sbw.quantize_fp8(x, codes=codes(4, 300), scales=scales(4, 2))
    with pytest.raises(ValueError, match="scales must be"):
        sbw.quantize_fp8(x, codes=codes(4, 300), scales=scales(4, 3, torch.float32))
    with pytest.raises(ValueError, match="block_rows"):
        sbw.quantize_fp8(x, block_rows=7)


def test_python_refusals_of_matmul(sbw):
    a, sa, b, sb = codes(4, 300), scales(4, 3), codes(200, 300), scales(2, 3)
    with pytest.raises(ValueError, match="current HIP device"):
        sbw.matmul_fp8(a, sa, b, sb)
    with pytest.raises(ValueError, match="same columns"):
        sbw.matmul_fp8(a, sa, codes(200, 299), sb)
    with pytest.raises(ValueError, match="a_scales"):
        sbw.matmul_fp8(a, scales(4, 2), b, sb)
    with pytest.raises(ValueError, match="b_scales"):
        sbw.matmul_fp8(a, sa, b, scales(3, 3))
    with pytest.raises(TypeError, match="one type"):
        sbw.matmul_fp8(a, sa, b, scales(2, 3, torch.float32))
    with pytest.raises(TypeError):
        sbw.matmul_fp8(a, scales(4, 3, torch.bfloat16), b, scales(2, 3, torch.bfloat16))
    with pytest.raises(TypeError):
        sbw.matmul_fp8(a, sa, b, sb, dtype=torch.float16)
    with pytest.raises(ValueError, match="out must be"):
        sbw.matmul_fp8(a, sa, b, sb, out=torch.zeros((4, 200)))
    with pytest.raises(ValueError, match="float8_e4m3fn"):
        sbw.matmul_fp8(a.view(torch.uint8), sa, b, sb)
    with pytest.raises(ValueError, match="float8_e4m3fn"):
        sbw.matmul_fp8(a.view(torch.uint8).view(torch.float8_e5m2), sa, b, sb)
    with pytest.raises(ValueError, match="unit stride"):
        sbw.matmul_fp8(codes(300, 4).t(), sa, b, sb)
    with pytest.raises(ValueError, match="no gradient"):
        sbw.matmul_fp8(a, scales(4, 3, torch.float32).requires_grad_(), b, scales(2, 3, torch.float32))


def test_python_refusals_of_the_layer(sbw):
    x, w = torch.zeros((4, 300)), torch.zeros((7, 300))
    with pytest.raises(ValueError, match="current HIP device"):
        sbw.linear_fp8(x, w)
    with pytest.raises(ValueError, match="same columns"):
        sbw.linear_fp8(x, w[:, :299])
    with pytest.raises(ValueError, match="one or more"):
        sbw.linear_fp8(x[:, :0], w[:, :0])
    with pytest.raises(TypeError):
        sbw.linear_fp8(x, w.half())
    with pytest.raises(TypeError):
        sbw.linear_fp8(x, w, dtype=torch.float16)
    with pytest.raises(ValueError, match="two-dimensional"):
        sbw.linear_fp8(x[None], w)
    with torch.autograd.forward_ad.dual_level():
        with pytest.raises(ValueError, match="tangent"):
            sbw.linear_fp8(torch.autograd.forward_ad.make_dual(x, x), w)


# --- the reference itself ------------------------------------------------------------------

def test_reference_codes_are_the_type_of_torch():
    every = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(every, ref.DECODED, equal_nan=True)
    rng = np.random.default_rng(1)
    v = np.concatenate([rng.standard_normal(50000) * 50, np.exp2(rng.uniform(-14, 8.8, 50000)), ref.POSITIVE,
                        (ref.POSITIVE[1:] + ref.POSITIVE[:-1]) / 2]).clip(-448, 448)
    v = np.concatenate([v, -v]).astype(np.float32)
    assert np.array_equal(torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy(), ref.encoded(v.astype(np.float64)))


def test_reference_scales():
    x = np.zeros((1, 640), np.float32)
    x[0, 0], x[0, 128], x[0, 256], x[0, 384] = 448, np.nextafter(np.float32(448), np.float32(500)), 3.4e38, 1e-45
    codes, s = ref.quantized(x, 1, True)
    assert s.tolist() == [[1.0, 2.0, 2.0 ** 120, 2.0 ** -127, 2.0 ** -127]]
    assert codes[0, 0] == 126 and codes[0, 128] == 118
    _, s = ref.quantized(x, 1, False)
    assert s[0, 0] == 1.0 and s[0, 3] == s[0, 4] == 2.0 ** -126
