"""Filtered sampling on the CPU: refusals before any HIP call; the definition's own filters."""
import ctypes
import math

import numpy as np
import pytest
import torch

import sample_reference as ref

OK, INVALID, GAMMA, DELTA, UNSUPPORTED, NO_DEVICE, HIP = range(7)
DUMMY = ctypes.c_void_p(0x1000)   # rejected before it could be used


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def call(lib, logits=DUMMY, dtype=0, B=2, V=8, stride=8, seeds=DUMMY, inv_ts=None, inv_t=1.0, ks=None, k=0, ps=None, p=1.0,
         mins=None, least=0.0, tokens=DUMMY, logprobs=DUMMY, ws=DUMMY):
    return lib.sbw_sample_tokens(logits, dtype, B, V, stride, seeds, inv_ts, inv_t, ks, k, ps, p, mins, least, tokens, logprobs,
                                 ws, None)


def test_refusals(sbw):
    lib = sbw.raw()
    assert call(lib, B=-1) == INVALID
    assert call(lib, V=-1) == INVALID
    assert call(lib, V=0, stride=0) == INVALID
    assert call(lib, stride=7) == INVALID
    for name in ("logits", "seeds", "tokens"):
        assert call(lib, **{name: None}) == INVALID, name
    for t in (0.0, -1.0, math.nan, math.inf):
        assert call(lib, inv_t=t) == INVALID, t
    assert call(lib, p=math.nan) == INVALID
    assert call(lib, least=math.nan) == INVALID
    assert call(lib, dtype=2) == UNSUPPORTED
    assert call(lib, V=1 << 32, stride=1 << 32) == UNSUPPORTED
    assert call(lib, B=1 << 62, stride=1 << 20) == UNSUPPORTED
    assert call(lib, B=0, logits=None, seeds=None, tokens=None) == OK
    if lib.sbw_sample_tokens_workspace(2, 8) > 0:
        assert call(lib, ws=None) == INVALID
    for sizes in ((0, 100), (5, 0), (-1, 5), (5, -1), (5, 1 << 32)):
        assert lib.sbw_sample_tokens_workspace(*sizes) == 0


def test_python_refusals(sbw):
    x, seeds = torch.zeros((3, 8)), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError, match="current HIP device"):
        sbw.sample_tokens(x, seeds)
    with pytest.raises(ValueError, match="seeds"):
        sbw.sample_tokens(x, seeds[:2])
    with pytest.raises(ValueError, match="seeds"):
        sbw.sample_tokens(x, seeds.int())
    for name, t in (("inv_temperature", torch.ones(2)), ("inv_temperature", torch.ones(3).double()), ("top_k", torch.ones(3)),
                    ("top_p", torch.ones(3, 1)), ("min_p", torch.ones(6)[::2])):
        with pytest.raises(ValueError, match=name):
            sbw.sample_tokens(x, seeds, **{name: t})
    with pytest.raises(TypeError):
        sbw.sample_tokens(x.half(), seeds)
    with pytest.raises(ValueError, match="tokens"):
        sbw.sample_tokens(x, seeds, tokens=torch.zeros(3, dtype=torch.int64))
    with pytest.raises(ValueError, match="workspace"):
        sbw.sample_tokens(x, seeds, workspace=torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError, match="no gradient"):
        sbw.sample_tokens(x.clone().requires_grad_(), seeds)
    with pytest.raises(ValueError, match="negated"):
        sbw.sample_tokens(torch._neg_view(x), seeds)


def test_reference_filters():
    row = np.log(np.array([0.1, 0.4, 0.05, 0.3, 0.15], np.float32))
    cols = lambda *f: ref.kept_columns(row, 1.0, *f)[0].tolist()   # noqa: E731
    assert cols(0, 1.0, 0.0) == [1, 3, 4, 0, 2]
    assert cols(2, 1.0, 0.0) == [1, 3]
    assert cols(0, 0.69, 0.0) == [1, 3] and cols(0, 0.71, 0.0) == [1, 3, 4]
    assert cols(2, 0.5, 0.0) == [1] and cols(2, 0.6, 0.0) == [1, 3]      # 0.4 of 0.7 is more than a half
    assert cols(0, 0.0, 0.0) == [1]
    assert cols(0, 1.0, 0.3) == [1, 3, 4] and cols(0, 1.0, 1.0) == [1]
    tied = np.zeros(10, np.float32)
    assert ref.kept_columns(tied, 1.0, 0, 0.5, 0.0)[0].tolist() == [0, 1, 2, 3, 4]
    assert ref.kept_columns(tied, 1.0, 7, 1.0, 0.5)[0].tolist() == list(range(7))
