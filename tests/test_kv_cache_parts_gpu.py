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


@pytest.mark.parametrize("G", [1, 3, 8])
@pytest.mark.parametrize("d", [32, 64, 96, 128, 160, 256])
@pytest.mark.parametrize("bits_v", [3, 4, 8])
@pytest.mark.parametrize("bits_k", [3, 4, 8])
def test_every_instance(bits_k, bits_v, d, G):
    """Every pair of bits with every head size that has an instance, and those without; one, two and four warps on a tile. Whole pairs and split ones."""
    Batch(730 + d + G, 2, d, (bits_k, bits_v), 16, [70, 0, 1300, 333], G=G, dtype="bf16" if G == 3 else "f16").check()
    Batch(731 + d + G, 1, d, (bits_k, bits_v), 48, [17], G=G).check()


def test_the_timed_mixed_case():
    """Keys of 4, values of 8 bits, 80 channels, eight query heads on a cached head, pages of 48 keys."""
    Batch(740, 4, 80, (4, 8), 48, [333, 0, 120, 250, 301], G=8).check()
