"""Products that take the 256 x 256 forms, on sizes whose form is asserted: every result against a product in fp32, and
sampled rows and columns against the definition in 64 bits."""
import pytest
import torch

import fp8_forms as forms
import fp8_reference as ref
from test_gpu_fp8 import DTYPES, SCALES, close, say

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def matrix(g, rows, K, block_rows, scales, odd_start=False):
    """(codes, scales) made on the device: rows padded to whole blocks with NaN; scales that start at no whole word."""
    blocks = forms.blocks_of(K)
    codes = torch.randint(0, 256, (rows, blocks * 128), generator=g, device="cuda", dtype=torch.uint8)
    codes[(codes & 127) == 127] = 0x31
    codes[:, K:] = 0x7F
    n = -(-rows // block_rows)
    s = torch.exp2(torch.randint(-20, 5, (n, blocks), generator=g, device="cuda").float())
    if scales == "f32":
        s *= torch.empty_like(s).uniform_(1.0, 2.0, generator=g)
    s = s.to(SCALES[scales])
    if odd_start:
        held = torch.empty(s.numel() + 1, dtype=s.dtype, device="cuda")
        held[1:] = s.view(-1)
        s = held[1:].view(n, blocks)
    return codes.view(torch.float8_e4m3fn)[:, :K], s


def values(codes, scales):
    rows, K = codes.shape
    s = scales.float().repeat_interleave(128, dim=1)[:, :K]
    return codes.float() * (s if s.shape[0] == rows else s.repeat_interleave(128, dim=0)[:rows])


def host(codes, scales, at):
    """The reference's form of some rows, a scale for each."""
    of_rows = scales[at] if scales.shape[0] == codes.shape[0] else scales[at // 128]
    return codes.contiguous().view(torch.uint8)[at].cpu().numpy(), of_rows.double().cpu().numpy()


def check(sbw, a, b, dtype, what):
    got = sbw.matmul_fp8(*a, *b, dtype=DTYPES[dtype])
    M, K = a[0].shape
    N = b[0].shape[0]
    # All results, 4096 columns at a time.  The product in fp32 is off by u K of the magnitudes' sum, the kernel's by twice that (as it
    # may cut off instead of rounding); of each eight products seven lose 2^-13 of the largest at most, which is no more than
    # their sum.  (A block of 128 of K columns that is missing or counted twice changes a result by about sqrt(128) / K of it.)
    x = values(*a)
    for n in range(0, N, 4096):
        y = values(b[0][n:n + 4096], b[1][n:n + 4096] if b[1].shape[0] == N else b[1][n // 128:n // 128 + 32])
        want, size = x @ y.t(), x.abs() @ y.abs().t()
        tol = 3 * ref.U * (K + 8) * size
        if dtype == "bf16":
            tol += 7 * 2.0 ** -13 * size + 2.0 ** -8 * want.abs()
        off = (got[:, n:n + 4096].float() - want).abs()
        assert (off <= tol).all(), (what, n, (off / tol).max().item())
    rows = torch.unique(torch.tensor([0, 1, M // 2, M - 2, M - 1], device="cuda"))
    columns = torch.unique(torch.cat([torch.arange(0, 130), torch.arange(N // 2, N // 2 + 130), torch.arange(N - 130, N)])).cuda()
    want, tol = ref.product(*host(*a, rows), *host(*b, columns), dtype == "bf16")
    close(got[rows][:, columns], want, tol, what)
    return got


@pytest.mark.parametrize("M,N,K,inside,scales,dtype", forms.WIDE_SIZES)
def test_wide_products(sbw, M, N, K, inside, scales, dtype):
    assert forms.plan_of(M, N, K, inside, True)[0] == "256"
    assert inside == (scales == "e8m0" and dtype == "bf16")
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    for rows_b, odd_start in ((1, False), (128, True)):
        say(f"wide product {M}x{N}x{K} {scales} {dtype} blocks {rows_b} odd_start={odd_start}")
        a, b = matrix(g, M, K, 1, scales, odd_start), matrix(g, N, K, rows_b, scales, odd_start)
        got = check(sbw, a, b, dtype, (M, N, K, rows_b))
        for _ in range(3):
            assert torch.equal(sbw.matmul_fp8(*a, *b, dtype=DTYPES[dtype]), got)      # the same bits each time
        out = torch.full((M, N + 3), 5.0, dtype=DTYPES[dtype], device="cuda")
        sbw.matmul_fp8(*a, *b, dtype=DTYPES[dtype], out=out[:, 1:N + 1])
        assert torch.equal(out[:, 1:N + 1], got) and (out[:, 0] == 5).all() and (out[:, N + 1:] == 5).all()


@pytest.mark.parametrize("M,N,K,inside,scales,dtype", [s for s in forms.WIDE_SIZES if s[0] < 1024 or s[2] == 32000])
def test_wide_scales_that_are_no_number(sbw, M, N, K, inside, scales, dtype):
    """They reach their rows' results and no others."""
    g = torch.Generator(device="cuda").manual_seed(K)
    a, b = matrix(g, M, K, 1, scales), matrix(g, N, K, 1, scales)
    a[1][M // 2, -1] = float("nan")
    b[1][N // 3, 0] = float("nan")
    b[1][N - 1, -1] = float("nan")
    want = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    want[M // 2] = True
    want[:, N // 3] = True
    want[:, N - 1] = True
    say(f"wide nan scales {M}x{N}x{K} {scales} {dtype}")
    assert torch.equal(sbw.matmul_fp8(*a, *b, dtype=DTYPES[dtype]).isnan(), want)


def test_wide_nan_codes(sbw):
    g = torch.Generator(device="cuda").manual_seed(1)
    M, N, K = 700, 17001, 1424
    assert forms.plan_of(M, N, K, True, True)[0] == "256"
    a, b = matrix(g, M, K, 1, "e8m0"), matrix(g, N, K, 128, "e8m0")
    a[0][M - 1, K - 1] = float("nan")
    b[0][300, 0] = float("nan")
    want = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    want[M - 1] = True
    want[:, 300] = True
    assert torch.equal(sbw.matmul_fp8(*a, *b).isnan(), want)
