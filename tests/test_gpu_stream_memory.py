"""Calls of the watermark on a busy stream that is not the current one, while the current one allocates and
writes: what a call allocates is not memory that the current stream still uses or is given meanwhile."""
import pytest
import torch

pytestmark = pytest.mark.gpu
KEY = 15485863


@pytest.fixture(scope="module")
def sbw():
    import paper_2609_03844_amd as sbw
    return sbw


def calls(sbw):
    g = torch.Generator(device="cuda").manual_seed(5)
    B, V, N, L = 48, 50257, 300, 400
    x = 3 * torch.randn((B, V), generator=g, device="cuda")
    prev = torch.randint(0, V, (B, 4), generator=g, device="cuda", dtype=torch.int32)
    seeds = torch.randint(0, 1 << 62, (B,), generator=g, device="cuda")
    texts = torch.randint(0, V, (N, L), generator=g, device="cuda", dtype=torch.int32)
    return {
        "argmax": lambda **kw: sbw.watermark_argmax(x, prev, KEY, 0.25, 2.0, **kw),
        "argmax_shard": lambda **kw: sbw.watermark_argmax_shard(x, prev, 1000, KEY, 0.25, 2.0, **kw),
        "argmax_noalloc": lambda **kw: sbw.watermark_argmax_noalloc(x[:16], prev[:16], KEY, 0.25, 2.0, **kw),
        "sample": lambda **kw: sbw.watermark_sample(x, prev, KEY, 0.25, 2.0, seeds, **kw),
        "sample_shard": lambda **kw: sbw.watermark_sample_shard(x, prev, 1000, KEY, 0.25, 2.0, seeds, **kw),
        "green_mask": lambda **kw: (sbw.green_mask(prev, V, KEY, 0.25, **kw),),
        "detect": lambda **kw: sbw.detect(texts, KEY, 0.25, **kw),
        "detect_ex": lambda **kw: sbw.detect_ex(texts, KEY, 0.25, **kw),
        "detect_unique": lambda **kw: sbw.detect_ex(texts, KEY, 0.25, ignore_repeated=True, **kw),
    }, 2 * sbw.argmax_workspace_size(B, V)


@pytest.mark.parametrize("raw", [False, True])
@pytest.mark.parametrize("name", ["argmax", "argmax_shard", "argmax_noalloc", "sample", "sample_shard", "green_mask",
                                  "detect", "detect_ex", "detect_unique"])
def test_memory_of_another_stream(sbw, name, raw):
    of_name, words = calls(sbw)
    call = of_name[name]
    want = call()
    busy, side = torch.randn(4096, 4096, device="cuda"), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(3):
        with torch.cuda.stream(side):
            for _ in range(10):
                busy = busy @ busy * 1e-3
        got = call(stream=side.cuda_stream if raw else side)
        kept = [torch.empty_like(t).fill_(7) for t in want for _ in range(2)]     # the sizes that a call allocates
        kept += [torch.empty(words // 2, dtype=torch.int64, device="cuda").fill_(-1) for _ in range(2)]
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a, b)
        del kept
