"""The operators of include/sbw_step.h at the limits of their arguments."""
import numpy as np
import pytest
import torch

import head_accuracy
import step_reference as ref
from test_gpu_step import DTYPES, close, given, packed, sbw, upstream  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 3])
@pytest.mark.parametrize("which", ["p", "l", "h", "plh"])
@pytest.mark.parametrize("inv_t,scale", [(3e38, 1.0), (3e38, 1e-30), (1e37, 100.0), (1e-37, 1e36)])
def test_gradient_of_extreme_products(sbw, dtype, n, which, inv_t, scale):  # noqa: F811
    """Factors and upstream gradients whose product passes fp32's range: infinite where the gradient is, and
    0 for the columns of probability 0."""
    rng = np.random.default_rng(21)
    B, V = 4, 3001
    x = -np.abs(np.round(4 * rng.standard_normal((B, V)))).astype(np.float32)
    x[1] -= 1
    x[1, 77] = 0                               # one alone
    x[2] = 0                                   # all alike
    tokens = given(rng, B, V, n)
    tokens[1, 0] = 77
    t = torch.from_numpy(x).to(DTYPES[dtype]).cuda()
    flat = torch.from_numpy(tokens[:, 0].copy() if n == 1 else tokens).cuda()
    r = sbw.token_logprobs(t, flat, inv_t)
    stats, H = r.stats.cpu().numpy(), r.entropy.cpu().numpy()
    up = [np.float32(scale) * u if u is not None else None for u in upstream(rng, B, n, which)]
    given_up = [u if u is not None else np.zeros((B, n) if i == 0 else B) for i, u in enumerate(up)]
    want, tol = ref.gradient(x, tokens, inv_t, stats, H, *given_up, bf16=dtype == "bf16")
    limit = float(torch.finfo(DTYPES[dtype]).max)
    assert not ((np.abs(want) > 0.98 * limit) & (np.abs(want) < 1.02 * limit)).any()   # of the inputs
    want = np.where(np.abs(want) > limit, np.copysign(np.inf, want), want)
    dev = [torch.from_numpy(u).cuda() if u is not None else None for u in up]
    if dev[0] is not None:
        dev[0] = dev[0].view(flat.shape)
    close(sbw.token_logprobs_grad(t, flat, r.stats, r.entropy, *dev, inv_t), want, tol, f"{which} n={n}")


def test_what_requires_a_gradient(sbw):  # noqa: F811
    """On the native path too: inputs that a call would drop the gradient of, and the calls that are right."""
    x = torch.randn(3, 50, device="cuda", requires_grad=True)
    h = torch.randn(3, 128, device="cuda").bfloat16().requires_grad_()
    codes = torch.zeros((5, 64), dtype=torch.uint8, device="cuda")
    scales = torch.ones((5, 1), device="cuda", requires_grad=True)
    for call in (lambda: sbw.head_logits(h, codes, scales.detach()), lambda: sbw.head_logits(h.detach(), codes, scales),
                 lambda: sbw.top_candidates(x, 4)):
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad():
            call()
    assert torch.equal(sbw.top_candidates(x, 4, with_values=False)[0], sbw.top_candidates(x.detach(), 4)[0])
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    r = sbw.token_logprobs(x, ids)
    assert r.logprobs.requires_grad
    d = sbw.token_logprobs_grad(x, ids, r.stats, None, torch.ones(3, device="cuda"))   # a leaf's, by hand
    assert not d.requires_grad
    r.logprobs.sum().backward()
    assert torch.equal(x.grad, d)


def test_tangents_are_refused(sbw):  # noqa: F811
    """A forward-mode tangent of any floating-point input, which no call carries, is named and not dropped."""
    x = torch.randn(3, 50, device="cuda")
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    h, codes = torch.randn(3, 128, device="cuda").bfloat16(), torch.zeros((5, 64), dtype=torch.uint8, device="cuda")
    scales = torch.ones((5, 1), device="cuda")
    r = sbw.token_logprobs(x, ids)
    g = torch.ones(3, device="cuda")
    calls = [(lambda a: sbw.token_logprobs(a, ids), x), (lambda a: sbw.top_candidates(a, 4), x),
             (lambda a: sbw.top_candidates(a, 4, with_values=False), x),
             (lambda a: sbw.head_logits(a, codes, scales), h), (lambda a: sbw.head_logits(h, codes, a), scales),
             (lambda a: sbw.token_logprobs_grad(a, ids, r.stats, None, g), x),
             (lambda a: sbw.token_logprobs_grad(x, ids, a, None, g), r.stats),
             (lambda a: sbw.token_logprobs_grad(x, ids, r.stats, None, a), g),
             (lambda a: sbw.token_logprobs_grad(x, ids, r.stats, a, None, g, g), r.entropy)]
    with torch.autograd.forward_ad.dual_level():
        for i, (call, t) in enumerate(calls):
            call(t)
            with pytest.raises(ValueError, match="tangent"):
                call(torch.autograd.forward_ad.make_dual(t, torch.ones_like(t)))
                print("call", i, "took a dual tensor", flush=True)


@pytest.mark.parametrize("raw", [False, True])
def test_backward_before_the_outputs_are_there(sbw, raw):  # noqa: F811
    """Upstream gradients that read no output of a call on another, busy stream: the backward pass waits for what
    the call left."""
    rng = np.random.default_rng(22)
    x = torch.randn(16, 4097, device="cuda")
    ids = torch.from_numpy(given(rng, 16, 4097, 1)[:, 0].copy()).cuda()
    up = [torch.randn(16, device="cuda") for _ in range(3)]
    side, busy = torch.cuda.Stream(), torch.randn(4096, 4096, device="cuda")

    def gradient(stream):
        z = x.clone().requires_grad_()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            work = busy
            for _ in range(10):
                work = work @ busy * 1e-3
        r = sbw.token_logprobs(z, ids, stream=stream)
        d, = torch.autograd.grad(r[:3], z, up)
        torch.cuda.synchronize()
        return d
    want = gradient(None)
    for _ in range(3):
        assert torch.equal(gradient(side.cuda_stream if raw else side), want)


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [1024, 2304, 4096])
def test_head_accuracy(sbw, K, group):  # noqa: F811
    """Nearer to the definition than weights held as 128 + q would come: bf16 holds 16 + q as exactly, and its sums
    lose three bits less."""
    rng = np.random.default_rng(K + group)
    codes, s, exact_s = packed(rng, 512, K, group, "f32")
    h = torch.from_numpy(rng.standard_normal((4, K)).astype(np.float32)).to(torch.bfloat16)
    out = sbw.head_logits(h.cuda(), torch.from_numpy(codes).cuda(), s).double().cpu().numpy()
    h = h.float().numpy()
    want, _ = ref.head(h, codes, exact_s)
    off, coarse = (head_accuracy.off(x, want) for x in (out, head_accuracy.simulated(h, codes, exact_s, 128)))
    print(f"K={K} group={group}: {off / ref.U:.2f} u, held as 128 + q {coarse / ref.U:.2f} u", flush=True)
    assert off < coarse


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("K", [512, 4224])
def test_head_rows_without_a_number(sbw, K, group, dtype):  # noqa: F811
    """A hidden state with an infinity or NaN, at any column, gives NaN for every row of the head; the others'
    logits are as without it."""
    rng = np.random.default_rng(K * group)
    codes, s, _ = packed(rng, 101, K, group, "bf16")
    codes = torch.from_numpy(codes).cuda()
    h = torch.from_numpy(rng.standard_normal((18, K)).astype(np.float32)).to(torch.bfloat16).cuda()
    want = sbw.head_logits(h, codes, s, dtype=DTYPES[dtype])
    bad = {1: (0, np.inf), 4: (K - 1, -np.inf), 7: (K // 2 + 5, np.nan), 16: (77, np.inf), 17: (300, -np.inf)}
    for row, (column, value) in bad.items():
        h[row, column] = value
    out = sbw.head_logits(h, codes, s, dtype=DTYPES[dtype])
    for b in range(18):
        assert torch.isnan(out[b]).all() if b in bad else torch.equal(out[b], want[b]), b


def test_negated_views(sbw):  # noqa: F811
    """Upstream gradients that torch hands over as lazily negated views (of one element, so contiguous) count with
    their sign, and direct calls refuse such views."""
    x = torch.randn(1, 50, device="cuda")
    ids = torch.tensor([7], dtype=torch.int32, device="cuda")
    zero = torch.zeros(1, device="cuda")

    def gradient(f):
        z = x.clone().requires_grad_()
        f(sbw.token_logprobs(z, ids)).sum().backward()
        return z.grad
    want = gradient(lambda r: -r.logprobs)
    got = gradient(lambda r: torch.complex(zero, r.logprobs).conj().imag)
    assert torch.equal(got, want)
    up = torch.complex(zero, zero + 1).conj().imag
    assert up.is_neg() and up.is_contiguous()
    r = sbw.token_logprobs(x, ids)
    with pytest.raises(ValueError, match="resolve_neg"):
        sbw.token_logprobs_grad(x, ids, r.stats, None, up)
    assert torch.equal(sbw.token_logprobs_grad(x, ids, r.stats, None, up.resolve_neg()), want)
    with pytest.raises(ValueError, match="resolve_neg"):
        sbw.top_candidates(up[None], 1)
