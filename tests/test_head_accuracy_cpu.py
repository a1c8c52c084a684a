"""The head's arithmetic in numpy against its definition."""
import numpy as np
import pytest
import torch

import head_accuracy
import step_reference as ref


@pytest.mark.parametrize("K,group", [(1024, 32), (1024, 128), (4096, 64)])
def test_offsets(K, group):
    """Exact for whole numbers with any offset; for others the smaller offset is nearer."""
    rng = np.random.default_rng(K - group)
    codes = rng.integers(0, 256, (256, K // 2)).astype(np.uint8)
    scales = rng.uniform(0.5, 1.5, (256, K // group)).astype(np.float32)
    h = rng.integers(-3, 4, (2, K)).astype(np.float32)
    ones = np.ones_like(scales)
    for offset in (16, 128):
        assert np.array_equal(head_accuracy.simulated(h, codes, ones, offset), ref.head(h, codes, ones)[0])
    h = torch.from_numpy(rng.standard_normal((4, K)).astype(np.float32)).to(torch.bfloat16).float().numpy()
    want, _ = ref.head(h, codes, scales)
    near, far = (head_accuracy.off(head_accuracy.simulated(h, codes, scales, o), want) for o in (16, 128))
    assert near < far
