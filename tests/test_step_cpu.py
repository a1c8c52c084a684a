"""include/sbw_step.h on the CPU: what it declares is exported, bad arguments are refused
before any HIP call, and it compiles as C11."""
import ctypes
import math
import os
import re
import subprocess

import numpy as np
import pytest

import step_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "sbw_step.h")
OK, INVALID, GAMMA, DELTA, UNSUPPORTED, NO_DEVICE, HIP = range(7)
DUMMY = ctypes.c_void_p(0x1000)   # rejected before it could be used


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


@pytest.fixture(scope="module")
def lib(sbw):
    return sbw.raw()


def test_declared_symbols_are_exported(sbw):
    text = open(HEADER).read()
    declared = set(re.findall(r"^(?:sbw_status_t|int64_t)\s+(sbw_[a-z_0-9]+)\s*\(", text, re.M))
    assert declared == set(sbw.EXPORTED_STEP)
    out = subprocess.run(["nm", "-D", "--defined-only", sbw.library_path()], capture_output=True,
                         text=True, check=True).stdout
    assert declared <= set(re.findall(r"\sT\s(sbw_\w+)$", out, re.M))
    # the library exports the two headers' functions and no other sbw_ symbol
    assert set(re.findall(r"\sT\s(sbw_\w+)$", out, re.M)) == declared | set(sbw.EXPORTED)


def test_header_compiles_as_c(tmp_path):
    src = tmp_path / "use.c"
    src.write_text('#include "sbw_step.h"\nint main(void) { return SBW_STEP_MAX_TOKENS == 1024 && '
                   "sbw_top_candidates_workspace(0, 5, 1) == 0 ? 0 : 1; }\n")
    exe = tmp_path / "use"
    libdir = os.path.join(ROOT, "paper_2609_03844_amd")
    rocm = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "lib")
    subprocess.run(["gcc", "-std=c11", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"),
                    str(src), "-o", str(exe), "-L", libdir, "-lsbw", f"-Wl,-rpath,{libdir}",
                    f"-Wl,-rpath,{rocm}", f"-Wl,-rpath-link,{rocm}"], check=True)
    assert subprocess.run([str(exe)], timeout=60).returncode == 0


def lp(lib, logits=DUMMY, dtype=0, B=2, V=8, stride=8, tokens=DUMMY, n=1, inv_t=1.0, top=0,
       logprobs=DUMMY, lse=DUMMY, entropy=DUMMY, stats=DUMMY, ids=DUMMY, tops=DUMMY, ws=DUMMY):
    return lib.sbw_token_logprobs(logits, dtype, B, V, stride, tokens, n, inv_t, top, logprobs, lse,
                                  entropy, stats, ids, tops, ws, None)


def test_token_logprobs_refusals(lib):
    assert lp(lib, B=-1) == INVALID
    assert lp(lib, V=-1) == INVALID
    assert lp(lib, V=0, stride=0) == INVALID
    assert lp(lib, stride=7) == INVALID
    assert lp(lib, logits=None) == INVALID
    assert lp(lib, tokens=None) == INVALID
    assert lp(lib, logprobs=None) == INVALID
    assert lp(lib, top=3, ids=None) == INVALID
    assert lp(lib, n=-1) == INVALID
    assert lp(lib, top=-1) == INVALID
    assert lp(lib, n=1025) == UNSUPPORTED
    assert lp(lib, top=1025) == UNSUPPORTED
    assert lp(lib, dtype=2) == UNSUPPORTED
    assert lp(lib, V=1 << 32, stride=1 << 32) == UNSUPPORTED
    assert lp(lib, B=1 << 62, stride=1 << 20) == UNSUPPORTED
    for t in (0.0, -1.0, math.nan, math.inf):
        assert lp(lib, inv_t=t) == INVALID, t
    assert lp(lib, B=0, logits=None, tokens=None, logprobs=None) == OK
    if lib.sbw_token_logprobs_workspace(2, 8, 0) > 0:
        assert lp(lib, ws=None) == INVALID


def grad(lib, logits=DUMMY, dtype=0, B=2, V=8, stride=8, tokens=DUMMY, n=1, stats=DUMMY, entropy=DUMMY,
         g=DUMMY, gl=None, gh=None, inv_t=1.0, out=ctypes.c_void_p(0x2000), out_stride=8):
    return lib.sbw_token_logprobs_grad(logits, dtype, B, V, stride, tokens, n, stats, entropy, g, gl, gh,
                                       inv_t, out, out_stride, None)


def test_token_logprobs_grad_refusals(lib):
    assert grad(lib, B=-1) == INVALID
    assert grad(lib, stride=7) == INVALID
    assert grad(lib, out_stride=7) == INVALID
    assert grad(lib, V=0, stride=0, out_stride=0) == INVALID
    assert grad(lib, logits=None) == INVALID
    assert grad(lib, stats=None) == INVALID
    assert grad(lib, out=None) == INVALID
    assert grad(lib, tokens=None) == INVALID
    assert grad(lib, gh=DUMMY, entropy=None) == INVALID
    assert grad(lib, out=DUMMY, out_stride=16) == INVALID     # in place with another stride
    assert grad(lib, n=-1) == INVALID
    assert grad(lib, n=1025) == UNSUPPORTED
    assert grad(lib, dtype=7) == UNSUPPORTED
    assert grad(lib, inv_t=math.nan) == INVALID
    assert grad(lib, B=1 << 62, out_stride=1 << 20) == UNSUPPORTED
    assert grad(lib, B=0, logits=None, stats=None, out=None) == OK


def cand(lib, logits=DUMMY, dtype=0, B=2, V=8, stride=8, offset=0, k=3, ids=DUMMY, values=DUMMY, ws=DUMMY):
    return lib.sbw_top_candidates(logits, dtype, B, V, stride, offset, k, ids, values, ws, None)


def test_top_candidates_refusals(lib):
    assert cand(lib, B=-1) == INVALID
    assert cand(lib, stride=7) == INVALID
    assert cand(lib, V=0, stride=0) == INVALID
    assert cand(lib, logits=None) == INVALID
    assert cand(lib, ids=None) == INVALID
    assert cand(lib, offset=-1) == INVALID
    assert cand(lib, k=0) == INVALID
    assert cand(lib, k=1025) == UNSUPPORTED
    assert cand(lib, dtype=-1) == UNSUPPORTED
    assert cand(lib, offset=(1 << 32) - 7) == UNSUPPORTED
    assert cand(lib, B=0, logits=None, ids=None) == OK
    if lib.sbw_top_candidates_workspace(2, 8, 3) > 0:
        assert cand(lib, ws=None) == INVALID


def head(lib, hidden=DUMMY, B=2, K=256, hs=256, codes=DUMMY, scales=DUMMY, sd=0, group=128, V=8, out=DUMMY,
         dtype=0, stride=8):
    return lib.sbw_head_logits(hidden, B, K, hs, codes, scales, sd, group, V, out, dtype, stride, None)


def test_head_logits_refusals(lib):
    assert head(lib, B=-1) == INVALID
    assert head(lib, V=-1) == INVALID
    assert head(lib, K=0) == INVALID
    assert head(lib, K=192) == INVALID                         # not a multiple of 128
    assert head(lib, hs=255) == INVALID
    assert head(lib, stride=7) == INVALID
    for name in ("hidden", "codes", "scales", "out"):
        assert head(lib, **{name: None}) == INVALID, name
    assert head(lib, group=16) == UNSUPPORTED
    assert head(lib, K=8320, hs=8320) == UNSUPPORTED
    assert head(lib, dtype=2) == UNSUPPORTED
    assert head(lib, sd=2) == UNSUPPORTED
    assert head(lib, B=0) == OK
    assert head(lib, V=0, stride=0) == OK


def test_sizes_of_nothing(lib):
    for f in (lib.sbw_token_logprobs_workspace, lib.sbw_top_candidates_workspace):
        assert f(0, 100, 5) == 0 and f(5, 0, 5) == 0 and f(-1, 100, 5) == 0 and f(5, -1, 5) == 0


# --- the reference itself ------------------------------------------------------------------

def test_reference_gradient_is_the_difference_quotient():
    rng = np.random.default_rng(3)
    V, n, inv_t = 23, 4, 1.25
    x = rng.standard_normal((1, V)) * 2
    tokens = np.array([[3, -1, 3, 22]])
    g, gl, gh = rng.standard_normal((1, n)), rng.standard_normal(1), rng.standard_normal(1)

    def loss(z):
        (lp_, lse_, H_, _, _), _ = ref.logprobs(z, tokens, inv_t)
        return (lp_ * g).sum() + (lse_ * gl).sum() + (H_ * gh).sum()
    (_, lse, H, _, _), _ = ref.logprobs(x, tokens, inv_t)
    stats = np.stack([x.max(axis=1), lse - x.max(axis=1) * inv_t], axis=1)
    d, _ = ref.gradient(x, tokens, inv_t, stats, H, g, gl, gh)
    for v in range(V):
        step = np.zeros_like(x)
        step[0, v] = 1e-6
        assert abs((loss(x + step) - loss(x - step)) / 2e-6 - d[0, v]) < 1e-7


def test_reference_order():
    x = np.array([1.0, np.nan, 2.0, -0.0, 0.0, np.inf, 2.0, np.nan, -np.inf], np.float32)
    assert ref.order(x).tolist() == [1, 7, 5, 2, 6, 0, 3, 4, 8]


def test_reference_weights():
    codes = np.array([[0x80, 0xF1]], np.uint8)
    assert ref.weights(codes, np.array([[2.0]])).tolist() == [[-16.0, 0.0, -14.0, 14.0]]
