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


class Repeated:
    """Sequences that name the same few pages again and again, so that a group's part is long without a cache as large. One head of 64 channels
    (or d), one cluster: K codes 0 but for the first key's. `count[j]`: how often physical key j comes in a sequence."""

    def __init__(self, n_seq, n, G, bits_v, d=64, pages=40, zero_v=None):
        import torch
        from paper_2304_01089_b200 import binding
        P = 64
        self.n, self.d, self.G, self.n_seq = n, d, G, n_seq
        self.top, self.z = (1 << bits_v) - 1, (1 << bits_v) // 4 if zero_v is None else zero_v
        self.s_k, self.s_v = 0.125, 0.25
        self.LK = binding.Layout(np.arange(d), [d], [self.s_k], [0], 4)
        self.LV = binding.Layout(np.arange(d), [d], [self.s_v], [self.z], bits_v)
        self.cache = binding.KvCache(self.LK, self.LV, 1, P)
        self.rng = np.random.default_rng(n)
        width = -(-n // P)
        row = np.concatenate([[0], 1 + np.arange(width - 1) % (pages - 1)]).astype(np.int32)
        self.table = torch.from_numpy(np.tile(row, (n_seq, 1))).cuda()
        key = row[np.arange(n) // P].astype(np.int64) * P + np.arange(n) % P
        self.count = np.bincount(key, minlength=pages * P).astype(np.float64)
        self.kq, self.vq = np.zeros((pages * P, d), np.int64), self.rng.integers(self.z, self.top + 1, size=(pages * P, d))
        self.pools = [torch.zeros((pages, b), dtype=torch.uint8, device="cuda") for b in (self.cache.k_page_bytes, self.cache.v_page_bytes)]
        self.lens = torch.full((n_seq,), n, dtype=torch.int32, device="cuda")

    def run(self, q, qk_scale):
        import torch
        from paper_2304_01089_b200 import binding
        for L, codes, bits, at in ((self.LK, self.kq, 4, 0), (self.LV, self.vq, self.LV.bits, 1)):
            rows = np.zeros((len(codes), L.K_pad), np.uint8)
            idx = L.padded_index()
            rows[:, idx >= 0] = codes[:, idx[idx >= 0]]
            dev = torch.from_numpy(binding.codes_pack_host(rows, bits)).cuda()
            other = torch.zeros((len(codes), (self.LV if at == 0 else self.LK).row_bytes), dtype=torch.uint8, device="cuda")
            pools = [p if i == at else torch.zeros_like(p) for i, p in enumerate(self.pools)]
            binding.kv_cache_write(self.cache, *((dev, other) if at == 0 else (other, dev)), torch.arange(len(codes), device="cuda"), *pools)
        out = torch.empty_like(q)
        binding.attention_paged(self.cache, q, *self.pools, self.table, self.lens, out, qk_scale, n_q_heads=self.G)
        return out.double().cpu().numpy().reshape(self.n_seq, self.G, self.d)


@pytest.mark.parametrize("bits_v", [3, 4, 8])
@pytest.mark.parametrize("G,n_seq", [(1, 2000), (8, 500)])
def test_a_key_far_ahead_does_not_swallow_the_others(G, n_seq, bits_v):
    """The first key is 15 to 21 nats ahead and its value is 0; the output is what 40000 others add up to. More than a thousand tiles of 32 keys
    to a group of warps.

    In units of the first key's probability, the others' are e = exp(-delta) each. Of the 1023 that may share its reference each is off by at most
    2^-30, the others by 2^-30 e; all by a factor of 1 +- E: the scores (at most delta log2(e) =: A, and equal for all others) have at most 8
    roundings, (8 A + 8) 2^-24, ex2 another 2^-22. A part empties its integers every 32 tiles, and a pair has three parts at most: fewer than
    64 additions of sums, 2^-24 each. Then one rounding to the output's type."""
    import torch
    n = 40000
    r = Repeated(n_seq, n, G, bits_v)
    r.kq[0], r.vq[0] = 15, r.z
    delta = r.rng.uniform(15.0, 21.0, size=(n_seq, G))
    q = torch.from_numpy(np.repeat(delta[:, :, None], r.d, 2).reshape(n_seq, -1)).half().cuda()
    delta = q.double().cpu().numpy().reshape(n_seq, G, r.d)[:, :, :1]
    scale = np.float32(1.0 / (r.d * 15 * r.s_k))
    got = r.run(q, float(scale))
    delta = delta * (float(scale) * (r.d * 15 * r.s_k))
    e = np.exp(-delta)
    V = r.s_v * (r.vq - r.z)
    others = r.count.copy()
    others[0] -= 1                                                             # (the first key itself; page 0 comes once)
    mass, total = (others[:, None] * V).sum(0), 1.0 + (n - 1) * e
    want = e * mass / total
    A = delta * 1.4427
    E = (8 * A + 8) * 2.0 ** -24 + 2.0 ** -22 + 64 * 2.0 ** -24
    lost = 1023 * 2.0 ** -30 + n * e * 2.0 ** -30
    bound = (lost * V.max() + E * e * mass) / total + want * (lost + E * n * e) / total + 8 * 2.0 ** -24 * want
    bound = 1.001 * bound + HALF_STEP["f16"] * np.maximum(want + bound, 2.0 ** -14)
    off = np.abs(got - want) - bound
    assert (off <= 0).all(), (float(off.max()), float((np.abs(got - want) / want).max()))


@pytest.mark.parametrize("bits_v", [3, 4, 8])
@pytest.mark.parametrize("G,n_seq", [(1, 2000), (8, 500)])
def test_parts_of_more_than_a_thousand_tiles(G, n_seq, bits_v):
    """Probabilities as near to the largest integer as scores can bring them, and the largest codes: the first tile's keys have score 0, all others one
    just below the two powers of two of room that the reference leaves above it. Nothing may overflow between two flushes, and the sums of a whole part stay
    what they are: with V's codes all at their largest the output is that value."""
    import torch
    n = 40000
    r = Repeated(n_seq, n, G, bits_v, zero_v=1)
    r.kq[:] = 15
    r.kq[:32] = 0
    r.vq[:] = r.top
    scale = np.float32(1.0 / (r.d * 15 * r.s_k * 1.4426950408889634))
    for power in (1.999, 0.999, 3.999):                                         # room of the integers: 2, 1, 4 powers of two
        q = torch.full((n_seq, G * r.d), power, device="cuda").half()
        got = r.run(q, float(scale))
        want = r.s_v * (r.top - r.z)
        assert (np.abs(got - want) <= (HALF_STEP["f16"] + 8 * 2.0 ** -24) * want).all()
    # half of the keys at each end of the codes
    r.vq[::2] = 0
    got = r.run(q, float(scale))
    w = np.where(np.arange(len(r.count)) < 32, 2.0 ** -float(q[0, 0].double()), 1.0) * r.count
    w = w / w.sum()
    V = r.s_v * (r.vq[:, 0] - r.z)
    want = float((w * V).sum())
    # the ratio of the two probabilities is off by (8 A + 8) 2^-24 + 2^-22, A = 4; 2^-29 of each probability; additions as above
    bound = (2 * (40 * 2.0 ** -24 + 2.0 ** -22) + 2 * 2.0 ** -29 + 64 * 2.0 ** -24) * float((w * np.abs(V)).sum())
    assert (np.abs(got - want) <= bound + HALF_STEP["f16"] * (abs(want) + bound)).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits", [(3, 4), (4, 8), (8, 3), (4, 4)])
@pytest.mark.parametrize("G,lens", [(1, [5000, 1, 700]), (4, [333, 3001]), (9, [77, 1500])])
def test_within_the_roundings_of_the_sums(G, lens, bits, dtype):
    """Random batches against a bound without the generous terms of Batch.want.

    Scores: the products with integers are exact. A query's integer is one rounding of q s (2^-24) and one to the integer: the largest of a head lies
    in [2^29, 2^30), so 2^-30 of it with 8 bits, 8 / 2^29 where a step is 16 (4 bits), 32 / 2^29 where it is 64 (3 bits). Five more roundings
    of the sum. Probabilities: the argument of ex2 is rounded once more, ex2 is good to 2^-22, the integer to 2^-30 of the largest. Sums: one rounding
    each time the integers are emptied (every 32 tiles, or scaled by at most 1/8 before) and two a part and a run in the joins."""
    b = Batch(900 + G, 2, 96, bits, 16, lens, G=G, dtype=dtype)
    got = b.run().double().cpu().numpy().reshape(len(lens), 2, G, 96)
    s, d, at = b.site, 96, 0
    q = b.q.double().cpu().numpy().reshape(len(lens), 2, G, d)
    top_k, top_v = (1 << bits[0]) - 1, (1 << bits[1]) - 1
    centre = np.clip(s.v.z, 0, top_v)
    step = {3: 2.0 ** -24, 4: 2.0 ** -26, 8: 2.0 ** -30}[bits[0]]
    for i, n in enumerate(lens):
        kq, vq = b.kq[at:at + n], b.vq[at:at + n]
        at += n
        K, V = s.k.values(kq).reshape(n, 2, d), s.v.values(vq).reshape(n, 2, d)
        S = b.qk_scale * 1.4426950408889634 * np.einsum("hgd,nhd->hgn", q[i], K)
        P = np.exp2(S - S.max(-1, keepdims=True))
        total = P.sum(-1, keepdims=True)
        want = np.einsum("hgn,nhd->hgd", P / total, V)
        x = b.qk_scale * 1.4427 * np.abs(q[i] * s.k.s.astype(np.float64).reshape(2, 1, d))
        A = x.sum(-1, keepdims=True) * top_k
        E = 6 * 2.0 ** -24 * A + d * step * x.max(-1, keepdims=True) * top_k
        E = E + (S.max(-1, keepdims=True) - S + 4) * 2.0 ** -24 + 2.0 ** -22
        E = np.expm1(E * 0.6932)
        reach = np.abs(s.v.s.astype(np.float64) * (vq - centre)).reshape(n, 2, d)
        K_sums = n / 1024 + 2 * min(GROUPS, n / 32 + 1) + 16
        top = reach.max(0)[:, None, :]
        mean = want - (s.v.s.astype(np.float64) * (centre - s.v.z)).reshape(2, 1, d)
        num = np.einsum("hgn,nhd->hgd", P * (E + K_sums * 2.0 ** -24), reach) / total + n * 2.0 ** -30 / total * top
        den = ((P * (E + K_sums * 2.0 ** -24)).sum(-1, keepdims=True) + n * 2.0 ** -30) / total * np.abs(mean)
        bound = 1.01 * (num + den) + 6 * 2.0 ** -24 * (np.abs(mean) + np.abs(want))
        bound = bound + HALF_STEP[dtype] * np.maximum(np.abs(want) + bound, 2.0 ** -14 if dtype == "f16" else 0.0)
        off = np.abs(got[i] - want) - bound
        assert (off <= 0).all(), (i, float(off.max()))
