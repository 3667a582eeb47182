"""rptq_attention_paged where a pair's keys lie with many groups of warps: parts, runs of parts and their joins."""
import numpy as np
import pytest

from paged_cases import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits,d", [((4, 4), 128), ((3, 8), 96), ((8, 3), 256)])
@pytest.mark.parametrize("G", [1, 2, 5])
def test_runs_of_parts_are_joined_once_each(G, bits, d):
    """One pair of cached head and queries over all groups: hundreds of parts in runs of eight to forty. Every key has the same score, so
    every part counts as much as another, and one that were added twice or left out would show."""
    import torch
    b = Batch(700 + G, 1, d, bits, 64, [41003], G=G)
    b.q[:] = 0.0
    out = b.check()
    for _ in range(20):
        assert torch.equal(b.run(), out)
    b.q.normal_()
    out = b.check()
    for _ in range(20):
        assert torch.equal(b.run(), out)
