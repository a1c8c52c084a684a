"""Filtered sampling on the GPU against its definition."""
import numpy as np
import pytest
import torch

import oracle
import sample_reference as ref
from test_gpu_fp8 import layer_reference
from test_gpu_step import DTYPES, logits, placed, special

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def say(text):
    print(text, flush=True)


def new_seeds(rng, B):
    s = rng.integers(0, 2 ** 63, B, dtype=np.int64)
    return s, torch.from_numpy(s).cuda()


def check(sbw, t, exact, rng, inv_t=1.0, top_k=0, top_p=1.0, min_p=0.0, what="", seeds=None):
    """Parameters are numbers, or arrays with one for each row."""
    B = exact.shape[0]
    host, device = new_seeds(rng, B) if seeds is None else seeds

    def given(v, dtype):
        return torch.from_numpy(np.asarray(v).astype(dtype)).cuda() if isinstance(v, np.ndarray) else v
    tokens, logprobs = sbw.sample_tokens(t, device, given(inv_t, np.float32), given(top_k, np.int32),
                                         given(top_p, np.float32), given(min_p, np.float32))
    assert tokens.dtype == torch.int32 and logprobs.dtype == torch.float32
    tokens, logprobs = tokens.cpu().numpy(), logprobs.double().cpu().numpy()
    for b in range(B):
        of_row = [v[b] if isinstance(v, np.ndarray) else v for v in (inv_t, top_k, top_p, min_p)]
        answers = ref.sample(exact[b], np.uint64(host[b]), *of_row)
        fits = [a for a in answers if a[0] == tokens[b]]
        assert fits, (what, b, of_row, tokens[b], answers)
        assert any(np.array_equal(lp, logprobs[b], equal_nan=True) or abs(lp - logprobs[b]) <= tol for _, lp, tol in fits), \
            (what, b, of_row, logprobs[b], fits)
    return tokens


SIZES = [(1, 1), (13, 2), (13, 3), (3, 7), (13, 64), (26, 255), (26, 1000), (26, 2049), (26, 8192), (13, 20011), (26, 32001)]
FILTERS = [dict(), dict(top_k=1), dict(top_k=50, top_p=0.95, inv_t=1.25), dict(top_p=0.9), dict(top_p=0.5, inv_t=0.7),
           dict(min_p=0.05), dict(top_p=0.99, min_p=0.02, inv_t=2.0), dict(top_k=300), dict(top_k=1024, top_p=0.999),
           dict(top_k=1500, top_p=0.9), dict(top_p=1e-9), dict(min_p=1.0), dict(top_p=0.0, min_p=7.0), dict(min_p=1e-30)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,V", SIZES)
def test_filters_on_rows_of_all_kinds(sbw, B, V, dtype):
    rng = np.random.default_rng(B * 100000 + V)
    t, exact = placed(special(rng, B, V), dtype)
    for f in FILTERS:
        say(f"sample {dtype} {B}x{V} {f}")
        check(sbw, t, exact, rng, **f)


def requests(rng, B):
    kinds = [(1.25, 50, 0.95, 0.0), (1.0, 0, 0.9, 0.0), (1.0, 1, 1.0, 0.0), (1.0, 0, 1.0, 0.05), (0.5, 40, 1.0, 0.0),
             (1.0, 0, 1.0, 0.0), (0.8, 0, 0.95, 0.02), (1.0, 2000, 0.99, 0.0), (3.0, -1, 1.5, -1.0), (1.0, 2 ** 31 - 1, 0.3, 0.2),
             (0.0, 5, 0.9, 0.0), (np.inf, 0, 0.9, 0.0), (np.nan, 0, 1.0, 0.0), (-1.0, 0, 1.0, 0.0), (1.0, 0, np.nan, np.nan)]
    return (np.array(v) for v in zip(*(kinds[i] for i in rng.integers(0, len(kinds), B))))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,V", [(90, 130), (120, 5003), (60, 32000), (16, 128259)])
def test_parameters_of_each_row(sbw, B, V, dtype):
    rng = np.random.default_rng(V)
    t, exact = placed(special(rng, B, V), dtype, 3, 1)
    for _ in range(3):
        inv_t, top_k, top_p, min_p = requests(rng, B)
        say(f"sample each {dtype} {B}x{V}")
        check(sbw, t, exact, rng, inv_t, top_k, top_p, min_p)
    check(sbw, t, exact, rng, 1.25, top_k, 0.9, min_p)                # some of them


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_flat_peaked_and_tied_rows(sbw, dtype):
    """Much kept and little kept; equal logits that the filters part by their columns."""
    rng = np.random.default_rng(8)
    V = 50021
    x = np.stack([0.3 * rng.standard_normal(V), np.zeros(V), np.full(V, -3.25), np.round(rng.standard_normal(V)),
                  np.where(np.arange(V) % 7 == 3, 5.0, 0.0), np.where(np.arange(V) == 40000, 30.0, 0.0),
                  np.arange(V) / V, -np.arange(V) / 1000.0, np.where(np.arange(V) > V - 900, 2.0, -1e30),
                  logits(rng, 1, V)[0], 0.4 * logits(rng, 1, V)[0], np.where(rng.random(V) < 0.999, -np.inf, 1.0)]).astype(np.float32)
    t, exact = placed(x, dtype)
    for f in (dict(), dict(top_p=0.9), dict(top_p=0.5), dict(top_p=0.999), dict(top_k=100), dict(top_k=1000, top_p=0.5),
              dict(top_k=20000), dict(top_k=20000, top_p=0.7), dict(min_p=0.5), dict(min_p=0.9999), dict(top_p=0.25, min_p=0.01),
              dict(inv_t=1e-20, top_p=0.5), dict(inv_t=1e20, top_p=0.5), dict(inv_t=1e-38), dict(inv_t=30.0, min_p=0.1)):
        say(f"sample flat {dtype} {f}")
        check(sbw, t, exact, rng, **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("B,V", [(1, 152064), (64, 128256), (3, 1000003), (300, 700), (70, 40000)])
def test_launch_shapes(sbw, B, V, dtype):
    rng = np.random.default_rng(B + V)
    x = logits(rng, B, V)
    x[::5] *= np.float32(0.4)
    t, exact = placed(x, dtype)
    rows = rng.permutation(B)[:12]
    for f in (dict(top_k=50, top_p=0.95), dict(top_p=0.9), dict(min_p=0.05), dict()):
        say(f"sample {dtype} {B}x{V} {f}")
        seeds, device = new_seeds(rng, B)
        whole, lp = sbw.sample_tokens(t, device, 1.0, f.get("top_k", 0), f.get("top_p", 1.0), f.get("min_p", 0.0))
        part = [int(r) for r in rows]
        got = check(sbw, t[part], exact[part], rng, seeds=(seeds[part], device[part].contiguous()), **f)
        assert np.array_equal(got, whole.cpu().numpy()[part])
        one, lp1 = sbw.sample_tokens(t[part[:1]], device[part[:1]].contiguous(), 1.0, f.get("top_k", 0), f.get("top_p", 1.0),
                                     f.get("min_p", 0.0))
        assert one[0] == whole[part[0]]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("pad,offset", [(1, 0), (0, 1), (3, 5), (8, 8)])
def test_layouts(sbw, dtype, pad, offset):
    rng = np.random.default_rng(pad * 10 + offset)
    for B, V in ((13, 5003), (120, 777)):
        t, exact = placed(special(rng, B, V), dtype, pad, offset)
        for f in (dict(top_k=20), dict(top_p=0.8), dict(min_p=0.1), dict()):
            say(f"layout {dtype} {B}x{V} pad={pad} offset={offset} {f}")
            check(sbw, t, exact, rng, **f)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_without_filters_it_is_the_sampler(sbw, dtype):
    rng = np.random.default_rng(4)
    for B, V in ((26, 32001), (5, 257), (40, 128256)):
        t, _ = placed(special(rng, B, V), dtype)
        _, seeds = new_seeds(rng, B)
        prev = torch.zeros(B, dtype=torch.int32, device="cuda")
        for inv_t in (1.0, 0.7, 3.0):
            want, _ = sbw.watermark_sample(t, prev, 15485863, 0.0, 0.0, seeds, inv_temperature=inv_t)
            assert torch.equal(sbw.sample_tokens(t, seeds, inv_t)[0], want)
            assert torch.equal(sbw.sample_tokens(t, seeds, inv_t, top_k=V, top_p=1.0, min_p=0.0)[0], want)
            each = torch.full((B,), inv_t, device="cuda")
            assert torch.equal(sbw.sample_tokens(t, seeds, each)[0], want)


def test_draws_follow_the_kept_probabilities(sbw):
    """60000 draws of one row: chi squared against softmax over the kept."""
    from scipy import stats
    rng = np.random.default_rng(17)
    V, n = 4001, 60000
    row = logits(rng, 1, V)[0]
    t = torch.from_numpy(row).cuda().expand(n, V).contiguous()
    for f in (dict(top_k=12), dict(top_p=0.8, inv_t=0.4), dict(min_p=0.08, inv_t=0.5), dict(top_k=40, top_p=0.9, min_p=0.02, inv_t=0.7)):
        _, seeds = new_seeds(rng, n)
        inv_t = f.pop("inv_t", 1.0)
        tokens, _ = sbw.sample_tokens(t, seeds, inv_t, **f)
        columns, e = ref.kept_columns(row, float(np.float32(inv_t)), f.get("top_k", 0), float(np.float32(f.get("top_p", 1.0))),
                                      float(np.float32(f.get("min_p", 0.0))))
        counts = np.bincount(tokens.cpu().numpy(), minlength=V)
        assert counts.sum() == counts[columns].sum()
        expected = n * e / e.sum()
        big = expected > 20
        chi = ((counts[columns][big] - expected[big]) ** 2 / expected[big]).sum()
        assert big.sum() >= 2 and stats.chi2.sf(chi, big.sum() - 1) > 1e-6, (f, chi, big.sum())


def test_given_tensors_and_parts(sbw):
    rng = np.random.default_rng(2)
    t, _ = placed(logits(rng, 9, 5003), "f32")
    _, seeds = new_seeds(rng, 9)
    want = sbw.sample_tokens(t, seeds, top_p=0.9)
    tokens, logprobs = torch.empty(9, dtype=torch.int32, device="cuda"), torch.empty(9, device="cuda")
    workspace = torch.full((sbw.sample_tokens_workspace_size(9, 5003) + 1,), -1, dtype=torch.int64, device="cuda")
    got = sbw.sample_tokens(t, seeds, top_p=0.9, tokens=tokens, logprobs=logprobs, workspace=workspace)
    assert got[0] is tokens and got[1] is logprobs
    assert torch.equal(tokens, want[0]) and torch.equal(logprobs, want[1])
    assert workspace[-1] == -1
    only, none = sbw.sample_tokens(t, seeds, top_p=0.9, with_logprobs=False)
    assert none is None and torch.equal(only, want[0])
    leaf = t.clone().requires_grad_()
    with pytest.raises(ValueError, match="no gradient"):
        sbw.sample_tokens(leaf, seeds)
    assert torch.equal(sbw.sample_tokens(leaf, seeds, top_p=0.9, with_logprobs=False)[0], want[0])
    empty = sbw.sample_tokens(t[:0], seeds[:0], top_p=0.9)
    assert empty[0].shape == (0,) and empty[1].shape == (0,)


def test_graph_replays(sbw):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((40, 30011), generator=g, device="cuda")
    seeds = torch.randint(0, 1 << 62, (40,), generator=g, device="cuda")
    top_k = torch.zeros(40, dtype=torch.int32, device="cuda")
    top_k[::3] = 40

    def step():
        return sbw.sample_tokens(x, seeds, 1.25, top_k, 0.9), sbw.sample_tokens(x, seeds, min_p=0.1)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for i in range(5):
        x.normal_(0.0, [4.0, 0.3, 2.0, 1.0, 3.0][i], generator=g)
        seeds.random_(0, 1 << 62, generator=g)
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        for a, b in zip(held, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_graphs_share_a_workspace(sbw):
    """Two graphs with one workspace, replayed in turn on one stream."""
    g = torch.Generator(device="cuda").manual_seed(2)
    inputs = [2 * torch.randn((B, V), generator=g, device="cuda") for B, V in ((5, 30011), (40, 20000))]
    seeds = [torch.randint(0, 1 << 62, (x.shape[0],), generator=g, device="cuda") for x in inputs]
    words = max(sbw.sample_tokens_workspace_size(*x.shape) for x in inputs)
    workspace = torch.empty(words, dtype=torch.int64, device="cuda")
    want = [sbw.sample_tokens(x, s, top_p=0.9) for x, s in zip(inputs, seeds)]
    outs = [(torch.empty_like(t), torch.empty_like(lp)) for t, lp in want]
    graphs = []
    torch.cuda.synchronize()
    for x, s, (t, lp) in zip(inputs, seeds, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            sbw.sample_tokens(x, s, top_p=0.9, tokens=t, logprobs=lp, workspace=workspace)
    for turn in (0, 1, 0, 0, 1, 1):
        outs[turn][0].fill_(-5), outs[turn][1].fill_(7.0)
        graphs[turn].replay()
        workspace.fill_(-1)
        torch.cuda.synchronize()
        assert torch.equal(outs[turn][0], want[turn][0]) and torch.equal(outs[turn][1], want[turn][1])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_more_rows_than_take_a_turn(sbw, dtype):
    """Long rows are sampled 512 at a time: parameters, seeds and results of later turns are their own rows'."""
    rng = np.random.default_rng(12)
    B, V = 1100, 4999
    t, exact = placed(special(rng, B, V), dtype, 1, 3)
    inv_t, top_k, top_p, min_p = requests(rng, B)
    seeds, device = new_seeds(rng, B)
    tokens, logprobs = sbw.sample_tokens(t, device, *(torch.from_numpy(v.astype(d)).cuda() for v, d in
                                         ((inv_t, np.float32), (top_k, np.int32), (top_p, np.float32), (min_p, np.float32))))
    tokens, logprobs = tokens.cpu().numpy(), logprobs.double().cpu().numpy()
    for b in [0, 1, 510, 511, 512, 513, 1022, 1023, 1024, 1025, 1099] + [int(b) for b in rng.permutation(B)[:60]]:
        answers = ref.sample(exact[b], np.uint64(seeds[b]), inv_t[b], top_k[b], top_p[b], min_p[b])
        assert any(a == tokens[b] and (np.array_equal(lp, logprobs[b], equal_nan=True) or abs(lp - logprobs[b]) <= tol)
                   for a, lp, tol in answers), (b, tokens[b], logprobs[b], answers)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [1, 5, 1025, 1100, 5003, 40001])
def test_top_k_of_every_size(sbw, V, dtype):
    """Around the sizes where another step takes over, of each row and of all."""
    rng = np.random.default_rng(V)
    sizes = np.array([0, 1, 2, 63, 64, 65, 255, 256, 257, 1023, 1024, 1025, V - 1, V, V + 1])
    x = 3 * rng.standard_normal((sizes.size, V)).astype(np.float32)
    x[1::3] = np.round(x[1::3])
    t, exact = placed(x, dtype, 1, 1)
    for f in (dict(), dict(top_p=0.95), dict(min_p=0.01)):
        say(f"sample top-k {dtype} {V} {f}")
        check(sbw, t, exact, rng, top_k=sizes, **f)
    for k in (64, 65, 1024, 1025):
        say(f"sample top-k {dtype} {V} {k}")
        check(sbw, t[:6], exact[:6], rng, top_k=k, top_p=0.9)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V", [130, 5003])
def test_scores_beyond_the_type(sbw, V, dtype):
    """Temperatures so low that scores overflow, so high that they vanish, and the smallest min-p."""
    rng = np.random.default_rng(V)
    x = rng.standard_normal((6, V)).astype(np.float32)
    x[1] = -np.abs(x[1]) - 2
    x[2] *= 1e-30
    x[3, 5:] = -np.inf
    x[4] = np.abs(x[4]) + 2
    x[5] *= 0.2
    t, exact = placed(x, dtype)
    seeds, device = new_seeds(rng, 6)
    for inv_t in (3.4e38, 2e38, 1e-45, 1e-38):
        for f in (dict(), dict(top_k=3), dict(top_k=400), dict(top_p=0.5), dict(min_p=0.5), dict(min_p=1e-45)):
            say(f"sample beyond {dtype} {V} {inv_t} {f}")
            tokens, logprobs = sbw.sample_tokens(t, device, inv_t, f.get("top_k", 0), f.get("top_p", 1.0), f.get("min_p", 0.0))
            tokens, logprobs = tokens.cpu().numpy(), logprobs.cpu().numpy()
            for b in range(6):
                answers = ref.sample(exact[b], np.uint64(seeds[b]), inv_t, **f)
                with np.errstate(over="ignore"):       # a log probability below all of fp32
                    assert any(a == tokens[b] and (np.float32(lp) == logprobs[b] or abs(lp - float(logprobs[b])) <= tol)
                               for a, lp, tol in answers), (b, tokens[b], logprobs[b], answers)


@pytest.mark.parametrize("raw", [False, True])
def test_another_stream(sbw, raw):
    """On a busy stream while the current one allocates and writes."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = 2 * torch.randn((48, 50257), generator=g, device="cuda")
    seeds = torch.randint(0, 1 << 62, (48,), generator=g, device="cuda")
    want = sbw.sample_tokens(x, seeds, top_p=0.9)
    busy, side = torch.randn(4096, 4096, device="cuda"), torch.cuda.Stream()
    words = max(1, sbw.sample_tokens_workspace_size(48, 50257))
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(10):
                busy = busy @ busy * 1e-3
        got = sbw.sample_tokens(x, seeds, top_p=0.9, stream=side.cuda_stream if raw else side)
        kept = [torch.empty_like(t).fill_(7) for t in want for _ in range(2)]
        kept += [torch.empty(words, dtype=torch.int64, device="cuda").fill_(-1) for _ in range(2)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        del kept


def test_in_a_decode_step(sbw):
    """A head in 8 bits, the watermark, filtered sampling, log probabilities: as they run together."""
    g = torch.Generator(device="cuda").manual_seed(6)
    B, V, K = 24, 20011, 512
    hidden = torch.randn((B, K), generator=g, device="cuda").to(torch.bfloat16)
    head = sbw.quantize_fp8(torch.randn((V, K), generator=g, device="cuda") / 8, 128)
    window = torch.randint(0, V, (B, 4), generator=g, device="cuda", dtype=torch.int32)
    seeds = torch.randint(0, 1 << 62, (B,), generator=g, device="cuda")
    raw = sbw.matmul_fp8(*sbw.quantize_fp8(hidden), *head, dtype=torch.float32)
    marked = raw.clone()
    sbw.watermark(marked, window, 15485863, 0.25, 2.0, "self_salt")
    expect = oracle.watermark_w(raw.cpu().numpy(), window.cpu().numpy(), 15485863, 0.25, 2.0, "self_salt")
    assert np.array_equal(marked.cpu().numpy(), expect)
    rng = np.random.default_rng(0)
    tokens = check(sbw, marked, expect, rng, 1.25, 50, 0.95, seeds=(seeds.cpu().numpy(), seeds))
    answer = sbw.token_logprobs(marked, torch.from_numpy(tokens).cuda(), 1.25)
    assert torch.isfinite(answer.logprobs).all()
    # the filters only raise the probability of what they keep
    _, lp = sbw.sample_tokens(marked, seeds, 1.25, 50, 0.95)
    assert (lp >= answer.logprobs - 1e-4).all()


def test_example_of_requests_and_an_8_bit_head(sbw):
    """The example's steps: tokens within what the filters keep, gradients against the layer's definition."""
    import importlib.util
    import pathlib
    path = pathlib.Path(__file__).resolve().parents[1] / "examples" / "decode_step.py"
    spec = importlib.util.spec_from_file_location("decode_step", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    g = torch.Generator(device="cuda").manual_seed(8)
    B, V, K = 12, 5003, 256
    hidden = torch.randn((B, K), generator=g, device="cuda").to(torch.bfloat16)
    weight = torch.randn((V, K), generator=g, device="cuda") * 3 / 16
    window = torch.randint(0, V, (B, 4), generator=g, device="cuda", dtype=torch.int32)
    seeds = torch.randint(0, 1 << 62, (B,), generator=g, device="cuda")
    full = lambda v: torch.full((B,), v, device="cuda")  # noqa: E731
    head = sbw.quantize_fp8(weight, 128)
    top_ks = torch.full((B,), 5, device="cuda", dtype=torch.int32)
    tokens, logprobs = example.requests_step(hidden, head, window, seeds, full(1.0), top_ks, full(0.9), full(0.0))
    logits = sbw.matmul_fp8(*sbw.quantize_fp8(hidden), *head)
    sbw.watermark(logits, window, example.KEY, example.GAMMA, example.DELTA)
    five = sbw.top_candidates(logits, 5)[0]
    assert (five == tokens[:, None]).any(1).all() and (logprobs <= 0).all()
    loss, of_hidden, of_weight = example.head_training_step(hidden, weight, tokens)
    # the layer's definition on the gradient of the log probabilities of its own logits, of type bf16
    z = sbw.linear_fp8(hidden, weight).double()
    p = torch.softmax(z, 1)
    p[torch.arange(B), tokens.long()] -= 1
    dy = (p / B).to(torch.bfloat16).float().cpu().numpy()
    want = layer_reference(hidden.float().cpu().numpy(), weight.cpu().numpy(), dy)
    # The kernel's gradient is within 2^-18 of this one, so one value in 2^8 at most rounds to another bf16, and its code moves by a
    # step of 2^-3 of it at most: sqrt(2^-8) 2^-3 = 2^-7 of the whole.  The results' own rounding is 2^-9.
    for got, name in ((of_hidden, "dx"), (of_weight, "dw")):
        exact, _ = want(name == "dx")[name]
        assert np.linalg.norm(got.double().cpu().numpy() - exact) < 2.0 ** -6 * np.linalg.norm(exact), name
