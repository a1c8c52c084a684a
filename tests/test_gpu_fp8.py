"""Matrices in 8-bit floating point, their products and the layer of them, on the GPU against their definitions."""
import numpy as np
import pytest
import torch

import fp8_reference as ref

pytestmark = pytest.mark.gpu
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
SCALES = {"e8m0": torch.float8_e8m0fnu, "f32": torch.float32}


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def say(text):
    print(text, flush=True)


def placed(x, dtype, pad=0, offset=0):
    """x [M, K] float32 -> (device tensor with padded, possibly unaligned rows, its exact values)."""
    M, K = x.shape
    buf = torch.full((M * (K + pad) + offset,), 7.0e4, dtype=dtype, device="cuda")
    t = buf[offset:].view(M, K + pad)[:, :K]
    t.copy_(torch.from_numpy(x))
    return t, t.float().cpu().numpy()


def bits(t):
    return t.contiguous().view(torch.uint8).cpu().numpy()


def same_codes(got, want):
    """Equal, a NaN as a NaN."""
    got, want = bits(got), np.asarray(want)
    nan = (want & 127) == 127
    assert np.array_equal((got & 127) == 127, nan)
    assert np.array_equal(got[~nan], want[~nan])


def special(rng, M, K):
    """Ordinary values with blocks out of the ordinary among them."""
    x = rng.standard_normal((M, K)).astype(np.float32)
    x *= np.exp2(rng.integers(-3, 4, (M, 1))).astype(np.float32)
    for j in range(0, K, 128):
        for i in range(M):
            kind = rng.integers(0, 24)
            part = x[i, j:j + 128]
            if kind == 0:
                part[:] = 0
            elif kind == 1:
                part *= np.float32(1e-38)
            elif kind == 2:
                part[:] = np.sign(part) * np.float32(448 * 2.0 ** int(rng.integers(-8, 9)))
            elif kind == 3:
                part *= np.float32(1e36)
            elif kind == 4:
                part[rng.integers(0, part.size)] = [np.nan, np.inf, -np.inf][rng.integers(0, 3)]
            elif kind == 5:
                part[:] = np.inf
            elif kind == 6:
                part[:] = np.float32(1e-45)
            elif kind == 7:
                part[:] = -0.0
            elif kind == 8:
                part[rng.integers(0, part.size)] = 3e38
    return x


SIZES = [(1, 1), (1, 127), (3, 128), (2, 129), (130, 5), (127, 300), (129, 256), (5, 2050), (260, 641), (33, 4099)]


@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,K", SIZES)
def test_quantize(sbw, M, K, dtype, scales):
    rng = np.random.default_rng(M * 10000 + K)
    for pad, offset in ((0, 0), (3, 1)):
        t, x = placed(special(rng, M, K), DTYPES[dtype], pad, offset)
        for block_rows in (1, 128):
            for transposed in (False, True):
                say(f"quantize {dtype} {scales} {M}x{K} rows={block_rows} transposed={transposed} pad={pad}")
                codes, s = sbw.quantize_fp8(t, block_rows, transposed, SCALES[scales])
                want, want_s = ref.quantized(x.T if transposed else x, block_rows, scales == "e8m0")
                assert s.dtype == SCALES[scales] and np.array_equal(s.double().cpu().numpy(), want_s)
                same_codes(codes, want)


def test_every_value_rounds_as_defined(sbw):
    """All bf16 magnitudes up to 448 beside a 448 that makes the scale 1; the halfway values among them."""
    x = torch.arange(0, 0x43E1, dtype=torch.int32).to(torch.int16).view(torch.bfloat16).float().numpy()
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-x.size % 127, np.float32)]).reshape(-1, 127)
    x = np.concatenate([np.full((x.shape[0], 1), 448.0, np.float32), x], axis=1)
    for scales in SCALES:
        codes, s = sbw.quantize_fp8(torch.from_numpy(x).cuda(), scale_dtype=SCALES[scales])
        assert (s.float() == 1).all()
        same_codes(codes, ref.encoded(x.astype(np.float64)))


def test_quantize_into_given_tensors(sbw):
    rng = np.random.default_rng(5)
    x = rng.standard_normal((37, 333)).astype(np.float32)
    t = torch.from_numpy(x).cuda()
    for transposed in (False, True):
        want, want_s = ref.quantized(x.T if transposed else x, 1, True)
        buf = torch.full((want.shape[0], want.shape[1] + 5), 3, dtype=torch.uint8, device="cuda")
        codes = buf.view(torch.float8_e4m3fn)[:, :want.shape[1]]
        scales = torch.empty(want_s.shape, dtype=torch.float8_e8m0fnu, device="cuda")
        got = sbw.quantize_fp8(t, transposed=transposed, codes=codes, scales=scales)
        assert got[0] is codes and got[1] is scales
        same_codes(codes, want)
        assert np.array_equal(scales.double().cpu().numpy(), want_s)
        assert (buf[:, want.shape[1]:] == 3).all()                  # behind the rows


def matrices(rng, rows, K, block_rows, scales, contiguous):
    """Codes and scales on the device and as the reference takes them."""
    codes = rng.integers(0, 256, (rows, K)).astype(np.uint8)
    codes[(codes & 127) == 127] = 0x31
    shape = (-(-rows // block_rows), -(-K // 128))
    if scales == "e8m0":
        s = np.exp2(rng.integers(-20, 5, shape)).astype(np.float32)
    else:
        s = (np.exp2(rng.uniform(-20, 5, shape))).astype(np.float32)
    width = K if contiguous else -(-K // 128) * 128
    held = torch.full((rows, width), 0x7F, dtype=torch.uint8, device="cuda")      # NaN behind the rows
    held[:, :K] = torch.from_numpy(codes)
    return held.view(torch.float8_e4m3fn)[:, :K], torch.from_numpy(s).cuda().to(SCALES[scales]), codes, s.astype(np.float64)


def close(got, want, tol, what):
    got = got.double().cpu().numpy()
    assert got.shape == want.shape, what
    assert np.array_equal(np.isnan(got), np.isnan(want)), what
    fine = np.isfinite(want)
    off = np.abs(got - want)[fine]
    bad = off > np.broadcast_to(tol, want.shape)[fine]
    assert not bad.any(), (what, off[bad][:5], np.broadcast_to(tol, want.shape)[fine][bad][:5])


PRODUCTS = [(1, 1, 1), (1, 5, 127), (2, 3, 128), (16, 300, 129), (17, 129, 257), (1, 1000, 2048), (33, 515, 1000),
            (64, 1024, 4096), (65, 256, 384), (130, 200, 512), (257, 300, 640), (128, 128, 2064), (300, 513, 272),
            (16, 64, 8192), (5, 2000, 656)]


@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("M,N,K", PRODUCTS)
def test_product(sbw, M, N, K, scales):
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    for rows_a, rows_b, contiguous, dtype in ((1, 1, True, "f32"), (1, 128, False, "bf16"), (128, 1, False, "f32"),
                                              (128, 128, True, "bf16")):
        say(f"product {scales} {M}x{N}x{K} blocks {rows_a} {rows_b} contiguous={contiguous} {dtype}")
        a, sa, a_, sa_ = matrices(rng, M, K, rows_a, scales, contiguous)
        b, sb, b_, sb_ = matrices(rng, N, K, rows_b, scales, contiguous)
        want, tol = ref.product(a_, sa_, b_, sb_, dtype == "bf16")
        got = sbw.matmul_fp8(a, sa, b, sb, dtype=DTYPES[dtype])
        assert got.dtype == DTYPES[dtype]
        close(got, want, tol, (M, N, K))
        pad = torch.full((M, N + 3), 5.0, dtype=DTYPES[dtype], device="cuda")
        sbw.matmul_fp8(a, sa, b, sb, dtype=DTYPES[dtype], out=pad[:, 1:N + 1])
        assert torch.equal(pad[:, 1:N + 1], got)                    # whatever the alignment
        assert (pad[:, 0] == 5).all() and (pad[:, N + 1:] == 5).all()


# many tiles, few tiles with long rows (parts of K), columns that end inside a block, blocks not a multiple of four
LARGE = [(512, 25700, 272), (513, 25601, 400), (1024, 4096, 8208), (300, 300, 8192), (40, 520, 4096), (64, 30000, 1040),
         (17, 130, 20000), (1000, 1000, 4112), (16, 70, 20000), (129, 40000, 528), (2, 100, 8320), (60, 3000, 1001),
         (1024, 600, 2003), (20, 30001, 777), (520, 26000, 200)]


@pytest.mark.parametrize("scales", ["e8m0", "f32"])
@pytest.mark.parametrize("M,N,K", LARGE)
def test_large_products(sbw, M, N, K, scales):
    rng = np.random.default_rng(M + N + K)
    rows = np.unique(np.concatenate([[0, M - 1], rng.integers(0, M, 6)]))
    columns = np.unique(np.concatenate([np.arange(min(N, 300)), np.arange(max(0, N - 300), N), rng.integers(0, N, 400)]))
    for rows_b, contiguous, dtype in ((1, True, "bf16"), (128, False, "bf16"), (128, False, "f32")):
        say(f"large product {scales} {M}x{N}x{K} blocks {rows_b} contiguous={contiguous} {dtype}")
        a, sa, a_, sa_ = matrices(rng, M, K, 1, scales, contiguous)
        b, sb, b_, sb_ = matrices(rng, N, K, rows_b, scales, contiguous)
        sb_ = ref.spread(sb_, N, K)[:, ::128]                       # a scale for each row
        want, tol = ref.product(a_[rows], sa_[rows], b_[columns], sb_[columns], dtype == "bf16")
        got = sbw.matmul_fp8(a, sa, b, sb, dtype=DTYPES[dtype])
        assert torch.isfinite(got).all()
        close(got[torch.from_numpy(rows).cuda()][:, torch.from_numpy(columns).cuda()], want, tol, (M, N, K))
        workspace = torch.full((sbw.matmul_fp8_workspace_size(M, N, K) + 1,), -1, dtype=torch.int64, device="cuda")
        again = torch.full((M, N + 8), 7.0, dtype=DTYPES[dtype], device="cuda")
        sbw.matmul_fp8(a, sa, b, sb, dtype=DTYPES[dtype], out=again[:, 3:3 + N], workspace=workspace)
        assert torch.equal(again[:, 3:3 + N], got) and workspace[-1] == -1
        assert (again[:, :3] == 7).all() and (again[:, 3 + N:] == 7).all()


def test_every_row_of_a_large_product(sbw):
    """Codes of one value a row, so that each result is known: no tile or part misses or repeats."""
    for M, N, K in ((600, 26000, 256), (1024, 4096, 8192), (48, 1000, 4096), (130, 513, 2048)):
        x = torch.exp2((torch.arange(M, device="cuda") % 5).float())[:, None].expand(M, K).contiguous()
        w = torch.exp2((torch.arange(N, device="cuda") % 7).float())[:, None].expand(N, K).contiguous()
        for scales in SCALES.values():
            a, b = sbw.quantize_fp8(x, scale_dtype=scales), sbw.quantize_fp8(w, scale_dtype=scales)
            for dtype in DTYPES.values():
                got = sbw.matmul_fp8(*a, *b, dtype=dtype).float()
                want = x[:, :1] * w[:, 0] * K
                assert ((got - want).abs() <= want * 2.0 ** -7).all(), (M, N, K, dtype)


@pytest.mark.parametrize("M", [1, 40, 200])
def test_product_of_nan_codes(sbw, M):
    rng = np.random.default_rng(M)
    for scales in SCALES:
        a, sa, a_, sa_ = matrices(rng, M, 400, 1, scales, False)
        b, sb, b_, sb_ = matrices(rng, 150, 400, 128, scales, False)
        a_[M // 2, 399] = b_[7, 0] = 0x7F
        a[M // 2, 399] = b[7, 0] = float("nan")
        want, tol = ref.product(a_, sa_, b_, sb_)
        close(sbw.matmul_fp8(a, sa, b, sb, dtype=torch.float32), want, tol, scales)


# --- the layer -------------------------------------------------------------------------------

def layer_reference(x, w, dy):
    """y, dx, dw of float32 values by the definition, each with its tolerance in fp32."""
    x8, w8, dy8 = ref.quantized(x, 1, True), ref.quantized(w, 128, True), ref.quantized(dy, 1, True)
    xt, wt, dyt = ref.quantized(x.T, 1, True), ref.quantized(w.T, 128, True), ref.quantized(dy.T, 1, True)
    return lambda bf16: {"y": ref.product(*x8, *w8, bf16), "dx": ref.product(*dy8, *wt, bf16), "dw": ref.product(*dyt, *xt, bf16)}


@pytest.mark.parametrize("x_type,w_type", [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (5, 130, 257), (200, 384, 256), (129, 65, 1000)])
def test_layer(sbw, M, N, K, x_type, w_type):
    rng = np.random.default_rng(M + N + K)
    x, x_ = placed(rng.standard_normal((M, K)).astype(np.float32), DTYPES[x_type], 3, 1)
    w, w_ = placed((rng.standard_normal((N, K)) / 16).astype(np.float32), DTYPES[w_type])
    x.requires_grad_(), w.requires_grad_()
    for dtype in (None, "f32", "bf16"):
        say(f"layer {M}x{N}x{K} {x_type} {w_type} {dtype}")
        y = sbw.linear_fp8(x, w, dtype=DTYPES[dtype] if dtype else None)
        y_type = dtype or x_type
        assert y.dtype == DTYPES[y_type]
        dy, dy_ = placed((rng.standard_normal((M, N)) * 1e-3).astype(np.float32), y.dtype, 5)
        dx, dw = torch.autograd.grad(y, (x, w), dy)
        want = layer_reference(x_, w_, dy_)
        close(y.detach(), *want(y_type == "bf16")["y"], "y")
        close(dx, *want(x_type == "bf16")["dx"], "dx")
        close(dw, *want(w_type == "bf16")["dw"], "dw")
        assert dx.dtype == x.dtype and dw.dtype == w.dtype
        # one side alone, and a gradient that is one value seen everywhere
        only, = torch.autograd.grad(sbw.linear_fp8(x.detach(), w, dtype=y.dtype), w, dy)
        assert torch.equal(only, dw)
        only, = torch.autograd.grad(sbw.linear_fp8(x, w.detach(), dtype=y.dtype), x, dy)
        assert torch.equal(only, dx)
        dx, dw = torch.autograd.grad(sbw.linear_fp8(x, w, dtype=y.dtype).sum(), (x, w))
        want = layer_reference(x_, w_, np.ones((M, N), np.float32))
        close(dx, *want(x_type == "bf16")["dx"], "dx of a sum")
        close(dw, *want(w_type == "bf16")["dw"], "dw of a sum")


def test_layer_gradient_is_the_difference_quotient(sbw):
    """Where every value is a small whole number the codes are exact and so is the layer: a step of 1 in one
    element changes the loss by its gradient."""
    rng = np.random.default_rng(11)
    M, N, K = 3, 5, 140
    x = torch.from_numpy(rng.integers(-7, 8, (M, K)).astype(np.float32)).cuda()
    w = torch.from_numpy(rng.integers(-7, 8, (N, K)).astype(np.float32)).cuda()
    g = torch.from_numpy(rng.integers(-7, 8, (M, N)).astype(np.float32)).cuda()

    def loss(x, w):
        return (sbw.linear_fp8(x, w) * g).sum()
    a, b = x.clone().requires_grad_(), w.clone().requires_grad_()
    dx, dw = torch.autograd.grad(loss(a, b), (a, b))
    for _ in range(20):
        m, n, k = rng.integers(0, M), rng.integers(0, N), rng.integers(0, K)
        step = x.clone()
        step[m, k] += 1
        assert (loss(step, w) - loss(x, w)).item() == dx[m, k].item()
        step = w.clone()
        step[n, k] += 1
        assert (loss(x, step) - loss(x, w)).item() == dw[n, k].item()


def test_layer_of_nothing(sbw):
    for M, N in ((0, 5), (4, 0), (0, 0)):
        x = torch.zeros((M, 130), device="cuda", requires_grad=True)
        w = torch.ones((N, 130), device="cuda", requires_grad=True)
        y = sbw.linear_fp8(x, w)
        assert y.shape == (M, N)
        dx, dw = torch.autograd.grad(y, (x, w), torch.zeros((M, N), device="cuda"))
        assert dx.shape == x.shape and dw.shape == w.shape and not dx.any() and not dw.any()
    codes, scales = sbw.quantize_fp8(torch.zeros((0, 5), device="cuda"))
    assert codes.shape == (0, 5) and scales.shape == (0, 1)
    assert sbw.matmul_fp8(codes, scales, codes, scales).shape == (0, 0)


def test_layer_keeps_its_codes(sbw):
    """What the caller writes into the inputs after the call does not reach the gradients."""
    x = torch.randn((40, 256), device="cuda").to(torch.bfloat16).requires_grad_()
    w = torch.randn((300, 256), device="cuda").to(torch.bfloat16).requires_grad_()
    dy = torch.randn((40, 300), device="cuda").to(torch.bfloat16)
    want = torch.autograd.grad(sbw.linear_fp8(x, w), (x, w), dy)
    y = sbw.linear_fp8(x, w)
    with torch.no_grad():
        x.zero_(), w.zero_()
    assert all(torch.equal(a, b) for a, b in zip(torch.autograd.grad(y, (x, w), dy), want))


def test_layer_in_front_of_log_probabilities(sbw):
    """A head's training step: layer, log probabilities, their gradient, the layer's."""
    g = torch.Generator(device="cuda").manual_seed(3)
    M, V, K = 70, 1003, 384
    x = torch.randn((M, K), generator=g, device="cuda").to(torch.bfloat16).requires_grad_()
    w = (torch.randn((V, K), generator=g, device="cuda") / 8).requires_grad_()
    tokens = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    y = sbw.linear_fp8(x, w, dtype=torch.float32)
    loss = -sbw.token_logprobs(y, tokens).logprobs.mean()
    loss.backward()
    z = y.detach().double()
    p = torch.softmax(z, 1)
    p[torch.arange(M), tokens.long()] -= 1
    want = layer_reference(x.detach().float().cpu().numpy(), w.detach().cpu().numpy(), (p / M).float().cpu().numpy())
    # codes of the gradient may differ by a step where a value lies between two: 2^-3 of the values is the largest step
    for got, name in ((x.grad, "dx"), (w.grad, "dw")):
        exact, _ = want(name == "dx")[name]
        off = np.linalg.norm(got.double().cpu().numpy() - exact) / np.linalg.norm(exact)
        assert off < 2.0 ** -8, (name, off)


# --- streams, graphs, devices ------------------------------------------------------------------

def test_graph_replays(sbw):
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((48, 520), generator=g, device="cuda")
    w = torch.randn((700, 520), generator=g, device="cuda")
    w8 = sbw.quantize_fp8(w, 128)

    def step():
        return sbw.matmul_fp8(*sbw.quantize_fp8(x), *w8), sbw.quantize_fp8(x, transposed=True)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        x.normal_(generator=g)
        graph.replay()
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(held[0], want[0])
        assert torch.equal(held[1][0].view(torch.uint8), want[1][0].view(torch.uint8))


@pytest.mark.parametrize("raw", [False, True])
def test_another_stream(sbw, raw):
    """On a busy stream while the current one allocates and writes."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((300, 1000), generator=g, device="cuda")
    w = torch.randn((700, 1000), generator=g, device="cuda")
    want_q = sbw.quantize_fp8(x)
    w8 = sbw.quantize_fp8(w, 128)
    want = sbw.matmul_fp8(*want_q, *w8)
    busy, side = torch.randn(4096, 4096, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(10):
                busy = busy @ busy * 1e-3
        at = side.cuda_stream if raw else side
        q = sbw.quantize_fp8(x, stream=at)
        got = sbw.matmul_fp8(*q, *w8, stream=at)
        kept = [torch.empty_like(got).fill_(7) for _ in range(4)]
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(q[0].view(torch.uint8), want_q[0].view(torch.uint8))
        del kept


def test_repeats_are_equal(sbw):
    g = torch.Generator(device="cuda").manual_seed(9)
    a = sbw.quantize_fp8(torch.randn((257, 4096), generator=g, device="cuda"))
    b = sbw.quantize_fp8(torch.randn((1030, 4096), generator=g, device="cuda"), 128)
    for dtype in DTYPES.values():
        first = sbw.matmul_fp8(*a, *b, dtype=dtype)
        assert all(torch.equal(sbw.matmul_fp8(*a, *b, dtype=dtype), first) for _ in range(5))


@pytest.mark.parametrize("scales", ["e8m0", "f32"])
def test_scales_that_are_no_number(sbw, scales):
    """They reach their rows' results and no others, in every form: also where blocks behind the last one are looked at."""
    rng = np.random.default_rng(2)
    for M, N, K in ((3, 140, 300), (40, 140, 1300), (70, 300, 650), (520, 26000, 200)):
        say(f"nan scales {scales} {M}x{N}x{K}")
        a, sa, *_ = matrices(rng, M, K, 1, scales, False)
        b, sb, *_ = matrices(rng, N, K, 1, scales, False)
        sa[M // 2, -1] = float("nan")
        sb[N // 3, 0] = float("nan")
        for dtype in DTYPES.values():
            got = sbw.matmul_fp8(a, sa, b, sb, dtype=dtype).isnan()
            want = torch.zeros((M, N), dtype=torch.bool, device="cuda")
            want[M // 2] = True
            want[:, N // 3] = True
            assert torch.equal(got, want)


def test_graphs_share_a_workspace(sbw):
    """Two graphs of products in parts of K with one workspace, replayed in turn on one stream."""
    g = torch.Generator(device="cuda").manual_seed(4)
    sizes = ((40, 300, 8192), (200, 300, 4096))
    pairs = [(sbw.quantize_fp8(torch.randn((M, K), generator=g, device="cuda")),
              sbw.quantize_fp8(torch.randn((N, K), generator=g, device="cuda"), 128)) for M, N, K in sizes]
    words = max(sbw.matmul_fp8_workspace_size(*s) for s in sizes)
    assert min(sbw.matmul_fp8_workspace_size(*s) for s in sizes) > 0
    workspace = torch.empty(words, dtype=torch.int64, device="cuda")
    want = [sbw.matmul_fp8(*a, *b) for a, b in pairs]
    outs, graphs = [torch.empty_like(w) for w in want], []
    torch.cuda.synchronize()
    for (a, b), out in zip(pairs, outs):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            sbw.matmul_fp8(*a, *b, out=out, workspace=workspace)
    for turn in (0, 1, 0, 0, 1, 1):
        outs[turn].fill_(7.0)
        graphs[turn].replay()
        workspace.fill_(-1)
        torch.cuda.synchronize()
        assert torch.equal(outs[turn], want[turn])


def test_layer_in_a_graph(sbw):
    """Forward and backward captured together and replayed with new inputs between; refused while an eager result lives."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = torch.randn((70, 384), generator=g, device="cuda").requires_grad_()
    w = torch.randn((500, 384), generator=g, device="cuda").requires_grad_()
    dy = torch.randn((70, 500), generator=g, device="cuda")

    def step():
        y = sbw.linear_fp8(x, w)
        return [y.detach(), *torch.autograd.grad(y, (x, w), dy)]
    eager = sbw.linear_fp8(x, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    refused = None
    marker = torch.zeros(8, device="cuda")
    with torch.cuda.graph(graph):
        marker.add_(1.0)                     # a graph of something
        try:
            sbw.linear_fp8(x, w)
        except RuntimeError as error:
            refused = str(error)
    assert refused is not None and "eager graph" in refused
    del eager
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(4):
        with torch.no_grad():
            x.normal_(generator=g), w.normal_(generator=g)
        dy.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, step()))


def test_layer_on_a_side_stream(sbw):
    """Its backward pass follows it there."""
    g = torch.Generator(device="cuda").manual_seed(6)
    x = torch.randn((70, 384), generator=g, device="cuda").to(torch.bfloat16).requires_grad_()
    w = torch.randn((500, 384), generator=g, device="cuda").requires_grad_()
    dy = torch.randn((70, 500), generator=g, device="cuda").to(torch.bfloat16)
    want = torch.autograd.grad(sbw.linear_fp8(x, w), (x, w), dy)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        y = sbw.linear_fp8(x, w)
        got = torch.autograd.grad(y, (x, w), dy)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
