"""rptq_attention_paged where rounding inside the sums shows: means near zero.

Bounds are derived beside each test. A part is what one group of warps works on; with one token a call there are at most 148 * 3 * 4 of them."""
import numpy as np
import pytest

from paged_cases import HALF_STEP, Batch

pytestmark = pytest.mark.gpu
GROUPS = 148 * 3 * 4


def _write_codes(b, kq, vq):
    """These codes into the batch's slots."""
    import torch
    from paper_2304_01089_b200 import binding
    rows = [torch.from_numpy(binding.codes_pack_host(t.code_rows(c), t.bits)).cuda() for t, c in zip((b.site.k, b.site.v), (kq, vq))]
    binding.kv_cache_write(b.site.cache, *rows, torch.from_numpy(b.slots).cuda(), *b.pools)
    b.kq, b.vq = kq, vq


@pytest.mark.parametrize("bits,d", [((4, 3), 128), ((4, 4), 128), ((4, 8), 128), ((8, 3), 72), ((3, 4), 40), ((3, 8), 200)])
@pytest.mark.parametrize("G", [1, 4])
def test_values_whose_mean_is_nearly_zero(G, bits, d):
    """Every key has the same probability, values come in pairs x, -x, and one key is left over with the smallest value there is: the mean is
    s / n. Sums of value codes are exact while they are integers; each part's sum is at most dev + 1 off zero, dev the largest code's distance
    from the zero point, so its rounding, its way through the joins (two levels: a product and a sum of two for each part and each run) and the
    quotient lose at most (parts + 16) 2^-24 (dev + 1) of one code, over n keys. Then one rounding to the output's type."""
    n = 60001
    b = Batch(800 + G, 2, d, bits, 64, [n, 77], G=G, dtype="bf16")
    s, top = b.site, (1 << bits[1]) - 1
    zero = s.v.z
    dev = np.clip(np.minimum(zero, top - zero), 0, None)                        # (zero points outside the codes: dev 0, all codes at the end nearest)
    rng = np.random.default_rng(0)
    at = np.clip(zero, 0, top)
    a = rng.integers(-dev, dev + 1, size=(n // 2, s.C))
    vq = np.empty((n, s.C), np.int64)
    vq[0:n - 1:2], vq[1::2] = at + a, at - a
    left = np.where(at < top, at + 1, at - 1)                                   # of the last key
    vq[n - 1] = left
    _write_codes(b, b.kq, np.concatenate([vq, b.vq[n:]]))
    b.q[:] = 0.0
    got = b.run().double().cpu().numpy()[0].reshape(2, G, d)
    scale = s.v.s.astype(np.float64).reshape(2, 1, d)
    inside = ((zero >= 0) & (zero <= top)).reshape(2, 1, d)
    want = scale * ((left - at) / n + (at - zero)).reshape(2, 1, d)             # (zero points outside: the rest is no difference of large numbers)
    parts = min(GROUPS, n // 32)
    bound = scale * (parts + 16) * 2.0 ** -24 * (dev.reshape(2, 1, d) + 1.0) / n + np.where(inside, 0.0, 8 * 2.0 ** -24) * np.abs(want)
    bound = bound + HALF_STEP["bf16"] * (np.abs(want) + bound)
    off = np.abs(got - want) - bound
    assert inside.any() and (off <= 0).all(), (float(off.max()), float((np.abs(got - want) / np.abs(want)).max()))
