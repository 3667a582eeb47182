"""rptq_kv_cache_write / _read and rptq_attention_paged against their definitions in 64 bits.

Codes are whole numbers decided from an exact product: they are equal. Values read back are s (q - z) rounded to fp32 and then to the
row's type, so numpy's fp32 product rounded the same way gives the same bits. Attention: tests/paged_cases.py derives the bound."""
import numpy as np
import pytest

from paged_cases import HALF_STEP, Batch, Site, torch_dtype

pytestmark = pytest.mark.gpu


def _slots(t):
    import torch
    return torch.from_numpy(np.asarray(t, np.int64)).cuda()


# ---------------------------------------------------------------- write and read
@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("bits", [(3, 3), (4, 4), (8, 8), (4, 8), (8, 3)])
@pytest.mark.parametrize("H,d,page", [(2, 64, 16), (3, 40, 48), (1, 256, 32), (2, 12, 16), (5, 128, 64), (4, 80, 16)])
def test_write_then_read(H, d, page, bits, dtype):
    import torch
    from paper_2304_01089_b200 import binding
    s = Site(100 + H * d + bits[0], H, d, bits, page)
    n_pages, n = 5, 37
    slots = s.rng.permutation(n_pages * page)[:n]
    slots[[3, 11]] = -1                                                    # skipped
    pools = s.pools(n_pages, 0x5A)
    before = s.read_codes(pools, np.arange(n_pages * page))
    dev, x = s.rows(n, dtype)
    binding.kv_cache_write(s.cache, *dev, _slots(slots), *pools)
    after = s.read_codes(pools, np.arange(n_pages * page))
    for t, b, a, rows in zip((s.k, s.v), before, after, x):
        want, keep = b.copy(), slots >= 0
        want[slots[keep]] = t.codes(rows)[keep]
        assert np.array_equal(a, want)
    back = [torch.full((n + 1, s.C), 7.0, dtype=torch_dtype(dtype), device="cuda") for _ in range(2)]
    binding.kv_cache_read(s.cache, *pools, _slots(slots), *back)
    for t, o, rows in zip((s.k, s.v), back, x):
        want = torch.from_numpy((t.codes(rows) - t.z).astype(np.float32) * t.s).to(torch_dtype(dtype))
        want[torch.from_numpy(slots < 0)] = 7.0                            # rows of negative slots are left as they were
        assert torch.equal(o[:n].cpu(), want) and bool((o[n] == 7.0).all())
    assert binding.get_device_status() == 0


@pytest.mark.parametrize("bits", [(3, 4), (4, 3), (8, 8)])
@pytest.mark.parametrize("first", [0, 1, 2, 3, 5, 14, 15])
@pytest.mark.parametrize("n", [1, 2, 3, 4, 5, 33])
def test_runs_of_slots_that_start_and_end_anywhere(first, n, bits):
    """A prompt's slots follow one another from any key of a page, across pages that do not."""
    from paper_2304_01089_b200 import binding
    s = Site(7 + first + n, 2, 96, bits, 16)
    pages = np.array([4, 1, 3, 0])
    logical = first + np.arange(n)
    slots = pages[logical // 16] * 16 + logical % 16
    pools = s.pools(6, 0xC3)
    before = s.read_codes(pools, np.arange(96))
    dev, x = s.rows(n)
    binding.kv_cache_write(s.cache, *dev, _slots(slots), *pools)
    after = s.read_codes(pools, np.arange(96))
    for t, b, a, rows in zip((s.k, s.v), before, after, x):
        b[slots] = t.codes(rows)
        assert np.array_equal(a, b)
    # in one call or a token at a time, the pool's bytes are the same
    again = s.pools(6, 0xC3)
    for i in range(n):
        binding.kv_cache_write(s.cache, dev[0][i:i + 1], dev[1][i:i + 1], _slots(slots[i:i + 1]), *again)
    assert all(bool((a == b).all()) for a, b in zip(pools, again))


def test_slots_in_any_order():
    from paper_2304_01089_b200 import binding
    s = Site(8, 3, 64, (4, 3), 32)
    for slots in (np.arange(63, -1, -1), np.repeat(np.arange(16), 4) * 4 + np.tile([1, 0, 3, 2], 16), np.arange(64) ^ 2, (np.arange(64) * 5) % 64):
        pools = s.pools(3, 0x99)
        dev, x = s.rows(64)
        binding.kv_cache_write(s.cache, *dev, _slots(slots), *pools)
        got = s.read_codes(pools, slots)
        for t, a, rows in zip((s.k, s.v), got, x):
            assert np.array_equal(a, t.codes(rows))


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("shift", [0, 1, 4])
def test_rows_that_lie_apart_and_off_their_alignment(dtype, shift):
    """K and V as slices of a wider matrix, as a fused projection gives them, from an element that need not be aligned."""
    import torch
    from paper_2304_01089_b200 import binding
    s = Site(9, 2, 64, (4, 4), 16)
    wide = torch.randn((21, 3 * s.C + 9), device="cuda").to(torch_dtype(dtype))
    k, v = wide[:, shift:shift + s.C], wide[:, s.C + shift:2 * s.C + shift]
    pools = s.pools(2)
    slots = np.arange(3, 24)
    binding.kv_cache_write(s.cache, k, v, _slots(slots), *pools)
    for t, a, rows in zip((s.k, s.v), s.read_codes(pools, slots), (k, v)):
        assert np.array_equal(a, t.codes(rows.double().cpu().numpy()))
    out = torch.full((21, 3 * s.C + 9), 3.0, device="cuda").to(torch_dtype(dtype))
    binding.kv_cache_read(s.cache, *pools, _slots(slots), out[:, shift:shift + s.C], out[:, s.C + shift:2 * s.C + shift])
    for i, (t, rows) in enumerate(zip((s.k, s.v), (k, v))):
        want = torch.from_numpy((t.codes(rows.double().cpu().numpy()) - t.z).astype(np.float32) * t.s).to(torch_dtype(dtype))
        assert torch.equal(out[:, i * s.C + shift:(i + 1) * s.C + shift].cpu(), want)
    assert bool((out[:, :shift] == 3.0).all()) and bool((out[:, 2 * s.C + shift:] == 3.0).all())


@pytest.mark.parametrize("bits", [(3, 8), (4, 4), (8, 3)])
@pytest.mark.parametrize("order", [0, 1])
def test_code_rows_in_and_out(bits, order):
    import torch
    from paper_2304_01089_b200 import binding
    s = Site(10, 3, 88, bits, 16, g=9, order=order)
    n = 29
    q = [s.rng.integers(0, 1 << t.bits, size=(n, s.C)) for t in (s.k, s.v)]
    rows = [torch.from_numpy(binding.codes_pack_host(t.code_rows(c), t.bits)).cuda() for t, c in zip((s.k, s.v), q)]
    slots = s.rng.permutation(48)[:n]
    pools = s.pools(3, 0xFF)
    binding.kv_cache_write(s.cache, *rows, _slots(slots), *pools)
    for a, c in zip(s.read_codes(pools, slots), q):
        assert np.array_equal(a, c)
    back = [torch.full_like(r, 0x77) for r in rows]
    binding.kv_cache_read(s.cache, *pools, _slots(slots), *back)
    assert all(torch.equal(a, b) for a, b in zip(back, rows))


def test_ties_ends_and_values_that_are_not_finite():
    import torch
    from paper_2304_01089_b200 import binding
    C = 64
    for bits in (3, 4, 8):
        L = binding.Layout(np.arange(C), [C], [0.25], [3], bits)           # steps of a quarter: halves are ties
        c = binding.KvCache(L, L, 1, 16)
        x = np.concatenate([(np.arange(58) - 20) * 0.125, [np.inf, -np.inf, np.nan, 1e30, -1e30, 65504.0]]).astype(np.float32)
        rows = torch.from_numpy(x[None]).cuda()
        pools = [torch.zeros((1, c.k_page_bytes), dtype=torch.uint8, device="cuda") for _ in range(2)]
        binding.kv_cache_write(c, rows, rows, _slots([5]), *pools)
        out = [torch.empty((1, C), device="cuda") for _ in range(2)]
        binding.kv_cache_read(c, *pools, _slots([5]), *out)
        top = (1 << bits) - 1
        q = np.clip(np.rint(x.astype(np.float64)[:58] * 4.0) + 3, 0, top)
        want = np.concatenate([q, [top, 0, 0, top, 0, top]])
        for o in out:
            assert np.array_equal(o.cpu().numpy()[0] * 4 + 3, want)


def test_zero_points_and_scales_far_from_the_codes():
    import torch
    from paper_2304_01089_b200 import binding
    C = 128
    zero = np.array([-(1 << 20), (1 << 20), 0, 2097151], np.int32)
    scale = np.array([1e-3, 3e-4, 1e20, 0.1], np.float32)
    L = binding.Layout(np.arange(C), [32] * 4, scale, zero, 8)
    c = binding.KvCache(L, L, 2, 16)
    s, z = np.repeat(scale, 32), np.repeat(zero, 32).astype(np.int64)
    q = np.random.default_rng(0).integers(0, 256, size=(16, C))
    x = (s.astype(np.float64) * (q - z)).astype(np.float32)
    rows = torch.from_numpy(x).cuda()
    pools = [torch.zeros((1, c.k_page_bytes), dtype=torch.uint8, device="cuda") for _ in range(2)]
    binding.kv_cache_write(c, rows, rows, _slots(np.arange(16)), *pools)
    out = [torch.empty((16, C), device="cuda") for _ in range(2)]
    binding.kv_cache_read(c, *pools, _slots(np.arange(16)), *out)
    inv = (1.0 / s.astype(np.float64)).astype(np.float32).astype(np.float64)
    want = np.clip(np.rint(x.astype(np.float64) * inv) + z, 0, 255)
    for o in out:
        assert np.array_equal(o.cpu().numpy(), (want - z).astype(np.float32) * s)


def test_slots_past_the_pool_are_skipped_and_recorded():
    import torch
    from paper_2304_01089_b200 import binding
    s = Site(11, 2, 32, (4, 4), 16)
    pools = s.pools(2, 0x11)
    keep = [p.clone() for p in pools]
    dev, _ = s.rows(3)
    assert binding.get_device_status() == 0
    binding.kv_cache_write(s.cache, *dev, _slots([32, 1 << 40, -7]), *pools)
    assert binding.get_device_status() == binding.ERR_BAD_SLOT
    assert all(torch.equal(a, b) for a, b in zip(pools, keep))
    out = [torch.full((3, s.C), 2.0, device="cuda") for _ in range(2)]
    binding.kv_cache_read(s.cache, *pools, _slots([-1, 1 << 62, 32]), *out)
    assert binding.get_device_status() == binding.ERR_BAD_SLOT
    assert all(bool((o == 2.0).all()) for o in out)
    binding.kv_cache_read(s.cache, *pools, _slots([-1, -1 << 62, 31]), *out)
    assert binding.get_device_status() == 0


def test_a_slot_may_be_read_any_number_of_times():
    import torch
    from paper_2304_01089_b200 import binding
    s = Site(12, 2, 64, (4, 3), 16)
    pools = s.pools(1)
    dev, x = s.rows(16)
    binding.kv_cache_write(s.cache, *dev, _slots(np.arange(16)), *pools)
    slots = np.array([3, 3, 3, 3, 0, 1, 2, 3, 4, 5, 9, 9, 8, 8, 15])
    for t, a, rows in zip((s.k, s.v), s.read_codes(pools, slots), x):
        assert np.array_equal(a, t.codes(rows)[slots])
    out = [torch.empty((len(slots), s.C), device="cuda") for _ in range(2)]
    binding.kv_cache_read(s.cache, *pools, _slots(slots), *out)
    for t, o, rows in zip((s.k, s.v), out, x):
        assert np.array_equal(o.cpu().numpy(), (t.codes(rows)[slots] - t.z).astype(np.float32) * t.s)


# ---------------------------------------------------------------- attention
@pytest.mark.parametrize("bits", [(3, 3), (4, 4), (8, 8), (4, 8), (8, 3), (3, 4)])
@pytest.mark.parametrize("lens", [[1], [16], [17], [31, 0, 33], [100, 1, 47, 48, 49]])
@pytest.mark.parametrize("d,page", [(64, 16), (128, 32), (80, 48), (256, 16)])
def test_attention_lengths_bits_heads(d, page, lens, bits):
    Batch(200 + d + len(lens), 2, d, bits, page, lens).check()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bits", [(3, 8), (4, 4), (8, 3)])
@pytest.mark.parametrize("G", [1, 2, 3, 4, 5, 8, 12, 17])
def test_attention_query_heads_that_share_a_cached_head(G, bits, dtype):
    Batch(300 + G, 2, 96, bits, 16, [70, 5, 0, 129], G=G, dtype=dtype).check()


@pytest.mark.parametrize("d", [4, 12, 32, 36, 100, 132, 160, 200, 224, 248])
@pytest.mark.parametrize("bits", [(3, 3), (4, 4), (8, 8)])
def test_attention_head_sizes(d, bits):
    Batch(400 + d, 2, d, bits, 16, [45, 64], G=3 if d % 8 else 1).check()


@pytest.mark.parametrize("bits", [(4, 4), (3, 3), (8, 8)])
@pytest.mark.parametrize("G", [1, 4, 8])
def test_attention_long_sequences_are_split(G, bits):
    Batch(500 + G, 1, 64, bits, 64, [9000], G=G).check()
    Batch(501 + G, 2, 128, bits, 16, [3001, 40, 2500], G=G, dtype="bf16").check()


@pytest.mark.parametrize("bits,G", [((4, 4), 1), ((8, 8), 8)])
def test_attention_one_head_over_a_very_long_sequence(bits, G):
    Batch(506, 1, 128, bits, 256, [70000], G=G).check()


def test_attention_many_sequences():
    rng = np.random.default_rng(3)
    Batch(510, 3, 64, (4, 4), 16, rng.integers(0, 200, size=300)).check()
    Batch(511, 1, 32, (8, 4), 32, rng.integers(0, 3, size=2000)).check()
    Batch(512, 40, 64, (3, 3), 16, rng.integers(1, 60, size=40)).check()


@pytest.mark.parametrize("G", [1, 3, 6])
def test_attention_scores_that_differ_widely(G):
    """Large queries: one key takes nearly all of the probability, and the running maximum moves many times."""
    for scale in (8.0, 60.0):
        Batch(520 + G, 2, 64, (4, 4), 16, [500, 77], G=G, q_scale=scale, dtype="bf16").check()


@pytest.mark.parametrize("G", [1, 4])
def test_attention_rising_scores(G):
    """Keys in the order of their scores: every tile's maximum is above the one before; and the reverse."""
    import torch
    from paper_2304_01089_b200 import binding
    for sign in (1.0, -1.0):
        b = Batch(530, 1, 64, (8, 8), 16, [700], G=G, q_scale=4.0)
        # every query head the same, so that one order of the keys rises for all of them
        b.q = b.q[:, :64].repeat(1, G).contiguous()
        q = b.q.double().cpu().numpy()[0, :64]
        order = np.argsort(sign * (b.site.k.values(b.kq) @ q), kind="stable")
        k = torch.from_numpy(b.site.k.values(b.kq)[order]).float().cuda()
        v = torch.from_numpy(b.site.v.values(b.vq)[order]).float().cuda()
        binding.kv_cache_write(b.site.cache, k, v, torch.from_numpy(b.slots).cuda(), *b.pools)
        b.kq, b.vq = b.kq[order], b.vq[order]
        b.check()


def test_attention_does_not_depend_on_what_lies_behind_a_sequence():
    import torch
    outs = []
    for fill in (0x00, 0xFF, 0x5A):
        outs.append([Batch(540 + i, 2, d, bits, 16, [37, 1, 16, 0, 99], G=G, fill=fill).check()
                     for i, (d, bits, G) in enumerate([(64, (4, 4), 1), (128, (3, 3), 2), (80, (8, 8), 4), (256, (4, 8), 8)])])
    for a, b, c in zip(*outs):
        assert torch.equal(a, b) and torch.equal(a, c)


def test_attention_pages_outside_the_pool_are_left_out_and_recorded():
    """(Every page number is compared with the pool's size before an address is formed from it.)"""
    from paper_2304_01089_b200 import binding
    for G in (1, 4):
        b = Batch(550, 2, 64, (4, 4), 16, [100, 64, 30], G=G)
        assert binding.get_device_status() == 0
        for page, bad in ((2, -1), (0, b.n_pages), (5, 2147483647)):
            c = Batch(550, 2, 64, (4, 4), 16, [100, 64, 30], G=G)
            c.table_dev[0, page] = bad
            got = c.run().double().cpu().numpy()
            assert binding.get_device_status() == binding.ERR_BAD_SLOT
            left = np.r_[0:100][np.r_[0:100] // 16 != page]
            c.kq, c.vq = np.concatenate([c.kq[left], c.kq[100:]]), np.concatenate([c.vq[left], c.vq[100:]])
            c.lens = [len(left), 64, 30]
            want, bound = c.want()
            assert (np.abs(got - want) <= bound).all()
        # all of a sequence's pages: nothing is left, zeros
        b.table_dev[1, :] = -5
        got = b.run()
        assert binding.get_device_status() == binding.ERR_BAD_SLOT
        assert not bool(got[1].any())


def test_attention_lengths_outside_the_table_are_clamped():
    import torch
    b = Batch(560, 2, 64, (4, 4), 16, [48, 48])
    want = b.run()
    b.lens_dev = torch.tensor([1 << 30, -3], dtype=torch.int32, device="cuda")
    got = b.run()
    assert torch.equal(got[0], want[0]) and not bool(got[1].any())


def test_attention_queries_that_are_not_finite():
    import torch
    for G in (1, 4):
        for bad in (float("nan"), float("inf"), -float("inf")):
            b = Batch(570, 2, 64, (4, 4), 16, [50, 200], G=G)
            want = b.run()
            b.q[1, 64 * G + 3] = bad                                        # a channel of sequence 1's query head G
            got = b.run()
            assert bool(torch.isnan(got[1, 64 * G:64 * G + 64]).all())
            got[1, 64 * G:64 * G + 64] = want[1, 64 * G:64 * G + 64]
            assert torch.equal(got, want)


def test_attention_queries_of_zero_and_of_extreme_size():
    import torch
    for G in (1, 4):
        for dtype, value in (("f16", 0.0), ("f16", 6e-8), ("f16", 65504.0), ("bf16", 1e-38), ("bf16", 1e30)):
            b = Batch(580, 1, 64, (4, 4), 16, [40], G=G, dtype=dtype)
            b.q[:] = value
            b.q[0, 1] = 0.0
            b.check()


def test_attention_scores_at_the_ends_of_their_range():
    """Scores far below -2^99 are scores like others; those that could pass 2^127 are refused as a query that is not finite is."""
    import torch
    for G in (1, 4):
        for bits in ((4, 4), (3, 3), (8, 8)):
            b = Batch(585, 1, 64, bits, 16, [40, 1], G=G, dtype="bf16")
            b.qk_scale = 1e30
            for sign in (1.0, -1.0):
                b.q[:] = sign
                out = b.run().double().cpu().numpy().reshape(2, G, 64)
                # the largest score is ahead of the others by far more than its rounding, and takes all: its value's row, rounded a few times
                K, V = b.site.k.values(b.kq), b.site.v.values(b.vq)
                S = 1e30 * sign * K[:40].sum(1)
                order = np.argsort(S)
                reach = 1e30 * np.abs(b.site.k.s.astype(np.float64)).sum() * ((1 << bits[0]) - 1)
                assert np.abs(S).max() < 2.0 ** 126 and S[order[-1]] - S[order[-2]] > 72 * 2.0 ** -24 * 1.4427 * reach + 1000
                reach_v = np.abs(b.site.v.s) * (np.abs(b.site.v.z) + (1 << bits[1]))
                for i, row in enumerate((V[order[-1]], V[40])):
                    assert (np.abs(out[i] - row) <= HALF_STEP["bf16"] * np.abs(row) + 8 * 2.0 ** -24 * reach_v).all()
            b.q[:, 0] = 1e38
            out = b.run()
            assert bool(torch.isnan(out[:, :64]).all()) and bool(torch.isfinite(out[:, 64:]).all())


def test_attention_is_the_same_every_time():
    import torch
    b = Batch(590, 2, 128, (4, 4), 16, [5000, 300, 1], G=2)
    first = b.run()
    for _ in range(5):
        assert torch.equal(b.run(), first)


def test_attention_row_distances_and_a_workspace_of_the_callers():
    import torch
    from paper_2304_01089_b200 import binding
    b = Batch(600, 2, 64, (4, 4), 16, [90, 33, 7])
    want = b.check()
    q = torch.full((3, 131), 9.0, dtype=torch.float16, device="cuda")
    q[:, 1:129] = b.q
    out = torch.full((4, 135), 5.0, dtype=torch.float16, device="cuda")
    table = torch.full((3, b.width + 3), -9, dtype=torch.int32, device="cuda")
    table[:, :b.width] = b.table_dev
    need = binding.attention_paged_workspace_bytes(b.site.cache, 2)
    ws = torch.full((need + 64,), 0xFF, dtype=torch.uint8, device="cuda")
    binding.attention_paged(b.site.cache, q[:, 1:129], *b.pools, table[:, :b.width], b.lens_dev, out[:, 3:131], b.qk_scale, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(out[:3, 3:131], want)
    assert bool((out[3] == 5.0).all()) and bool((out[:, :3] == 5.0).all()) and bool((out[:, 131:] == 5.0).all())
    assert bool((ws[need:] == 0xFF).all())


def test_pools_of_more_than_four_gibibytes():
    import torch
    from paper_2304_01089_b200 import binding
    b = Batch(610, 16, 128, (8, 8), 64, [200, 100])
    want = b.check()
    c = b.site.cache
    n_pages = (5 << 30) // c.k_page_bytes
    pools = [torch.zeros((n_pages, c.k_page_bytes), dtype=torch.uint8, device="cuda") for _ in range(2)]
    lift = n_pages - b.n_pages
    for p, small in zip(pools, b.pools):
        p[lift:] = small
    table = torch.where(b.table_dev >= 0, b.table_dev + lift, b.table_dev)
    out = torch.empty_like(b.q)
    binding.attention_paged(c, b.q, *pools, table, b.lens_dev, out, b.qk_scale)
    assert torch.equal(out, want)
    back = [torch.empty((300, b.site.C), dtype=torch.float16, device="cuda") for _ in range(4)]
    binding.kv_cache_read(c, *pools, torch.from_numpy(b.slots + lift * 64).cuda(), *back[:2])
    binding.kv_cache_read(c, *b.pools, torch.from_numpy(b.slots).cuda(), *back[2:])
    assert torch.equal(back[0], back[2]) and torch.equal(back[1], back[3])
    binding.kv_cache_write(c, back[1], back[0], torch.from_numpy(b.slots + lift * 64).cuda(), *pools)
    binding.kv_cache_write(c, back[1], back[0], torch.from_numpy(b.slots).cuda(), *b.pools)
    assert all(torch.equal(p[lift:], small) for p, small in zip(pools, b.pools))


# ---------------------------------------------------------------- as a server uses them
def test_on_other_streams_and_in_a_graph():
    """A decode step (write the new token, attend) captured once and replayed with new inputs and lengths, on its own stream."""
    import torch
    from paper_2304_01089_b200 import binding
    b = Batch(620, 2, 64, (4, 4), 16, [40, 17, 60], spare=4)
    s, side = b.site, torch.cuda.Stream()
    ws = torch.empty(binding.attention_paged_workspace_bytes(s.cache), dtype=torch.uint8, device="cuda")
    (k, v), _ = s.rows(3)
    slots, out = torch.full((3,), -1, dtype=torch.int64, device="cuda"), torch.empty_like(b.q)
    b.table = np.concatenate([b.table, np.full((3, 1), -1, np.int32)], 1)
    used = set(b.table[b.table >= 0].tolist())
    free = [p for p in range(b.n_pages) if p not in used]
    b.table_dev = torch.from_numpy(b.table).cuda()

    def step():
        binding.kv_cache_write(s.cache, k, v, slots, *b.pools)
        binding.attention_paged(s.cache, b.q, *b.pools, b.table_dev, b.lens_dev, out, b.qk_scale, workspace=ws)

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                                              # (slots are negative: nothing is written)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for turn in range(5):
        (nk, nv), x = s.rows(3)
        at = []
        for i, n in enumerate(b.lens):
            if n % 16 == 0:
                b.table[i, n // 16] = free.pop()
            at.append(int(b.table[i, n // 16]) * 16 + n % 16)
        ends = np.cumsum(b.lens)
        b.kq, b.vq = (np.insert(a, ends, t.codes(r), axis=0) for a, t, r in ((b.kq, s.k, x[0]), (b.vq, s.v, x[1])))
        b.lens = [n + 1 for n in b.lens]
        k.copy_(nk); v.copy_(nv); slots.copy_(torch.tensor(at)); b.table_dev.copy_(torch.from_numpy(b.table))
        b.lens_dev.copy_(torch.tensor(b.lens, dtype=torch.int32))
        b.q.copy_(torch.randn_like(b.q))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want, bound = b.want()
        assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()
    assert binding.get_device_status() == 0


@pytest.mark.parametrize("as_number", [False, True])
def test_a_workspace_that_the_call_allocates_belongs_to_its_stream(as_number, monkeypatch):
    """While the call waits on its stream, the current stream is not handed the memory of its workspace."""
    import torch
    from paper_2304_01089_b200 import binding
    b = Batch(623, 2, 128, (4, 4), 16, [5000, 70])
    want = b.check()
    need = binding.attention_paged_workspace_bytes(b.site.cache)
    at = []

    class Seen:
        def attention_paged(self, *args):
            at.append(args[9].data_ptr())
            return real.attention_paged(*args)

    real, side, out = binding._calls, torch.cuda.Stream(), torch.empty_like(b.q)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    monkeypatch.setattr(binding, "_calls", Seen())
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
    binding.attention_paged(b.site.cache, b.q, *b.pools, b.table_dev, b.lens_dev, out, b.qk_scale, stream=side.cuda_stream if as_number else side)
    mine = [torch.empty(need, dtype=torch.uint8, device="cuda").random_(0, 256) for _ in range(4)]
    assert at and not any(m.data_ptr() <= at[0] < m.data_ptr() + need or at[0] <= m.data_ptr() < at[0] + need for m in mine)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


def test_tables_of_no_pages():
    import torch
    from paper_2304_01089_b200 import binding
    b = Batch(624, 2, 64, (4, 4), 16, [20, 3])
    out = torch.full_like(b.q, float("nan"))
    binding.attention_paged(b.site.cache, b.q, *b.pools, b.table_dev[:, :0].contiguous(), b.lens_dev, out, b.qk_scale)
    assert not bool(out.any())
    assert binding.get_device_status() == 0


_FIRST = """
import numpy as np, torch
from paged_cases import Site
from paper_2304_01089_b200 import binding
s = Site(628, 2, 64, {bits}, 16)
pools = s.pools(30)
k, v = (torch.randn((450, s.C), dtype=torch.float16, device="cuda") for _ in range(2))
slots = torch.arange(450, device="cuda")
q = torch.randn((2, s.C * {G}), dtype=torch.float16, device="cuda")
table = torch.arange(30, dtype=torch.int32, device="cuda").reshape(2, 15)
lens = torch.tensor([240, 200], dtype=torch.int32, device="cuda")
out = [torch.zeros_like(q) for _ in range(2)]
back = [[torch.zeros_like(k) for _ in range(2)] for _ in range(2)]
ws = torch.empty(binding.attention_paged_workspace_bytes(s.cache, 2 * {G}), dtype=torch.uint8, device="cuda")
def call(i):
    binding.kv_cache_write(s.cache, k, v, slots, *pools)
    binding.kv_cache_read(s.cache, *pools, slots, *back[i])
    binding.attention_paged(s.cache, q, *pools, table, lens, out[i], 0.125, n_q_heads=2 * {G}, workspace=ws)
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    call(0)
for p in pools:
    p.zero_()
graph.replay()
torch.cuda.synchronize()
call(1)
torch.cuda.synchronize()
assert bool(out[1].any()) and torch.equal(out[0], out[1])
assert all(bool(y.any()) and torch.equal(x, y) for x, y in zip(*back))
assert binding.get_device_status() == 0
print("same")
"""


@pytest.mark.parametrize("bits, G", [((4, 4), 1), ((3, 8), 4)])
def test_first_calls_of_a_process_can_be_captured(bits, G):
    import os
    import subprocess
    import sys
    here = os.path.dirname(os.path.abspath(__file__))
    env = dict(os.environ, PYTHONPATH=os.pathsep.join([here, os.path.dirname(here), os.environ.get("PYTHONPATH", "")]))
    r = subprocess.run([sys.executable, "-c", _FIRST.format(bits=bits, G=G)], capture_output=True, text=True, timeout=300, env=env)
    assert r.returncode == 0 and r.stdout.split()[-1:] == ["same"], r.stderr[-2000:]


def test_two_graphs_that_share_a_workspace():
    """Captured over the same workspace and replayed by turns, with other work over it in between: what a call finds there does not matter."""
    import torch
    from paper_2304_01089_b200 import binding
    b = [Batch(625, 2, 128, (4, 4), 16, [5000, 70]), Batch(626, 1, 64, (8, 8), 32, [9000], G=4), Batch(627, 3, 96, (3, 3), 16, [700, 0, 33], G=2)]
    want = [x.check() for x in b]
    ws = torch.randint(0, 256, (max(binding.attention_paged_workspace_bytes(x.site.cache, x.site.H * x.G) for x in b),), dtype=torch.uint8, device="cuda")
    outs, graphs = [torch.empty_like(x.q) for x in b], []
    for x, o in zip(b, outs):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.attention_paged(x.site.cache, x.q, *x.pools, x.table_dev, x.lens_dev, o, x.qk_scale, n_q_heads=x.site.H * x.G, workspace=ws)
        graphs.append(g)
    for turn in range(6):
        if turn in (2, 4):
            ws.random_(0, 256)
        for i in ((0, 1, 2), (2, 1, 0), (1, 1, 0, 2))[turn % 3]:
            outs[i].fill_(float("nan"))
            graphs[i].replay()
            torch.cuda.synchronize()
            assert torch.equal(outs[i], want[i])
    assert binding.get_device_status() == 0


def test_two_calls_at_once():
    """Two streams with a workspace each, over the same pools."""
    import torch
    from paper_2304_01089_b200 import binding
    b = [Batch(630 + i, 2, 128, (4, 4), 16, [4000 - 100 * i, 50]) for i in range(2)]
    want = [x.check() for x in b]
    streams = [torch.cuda.Stream() for _ in b]
    ws = [torch.empty(binding.attention_paged_workspace_bytes(x.site.cache), dtype=torch.uint8, device="cuda") for x in b]
    outs = [[torch.empty_like(x.q) for _ in range(10)] for x in b]
    torch.cuda.synchronize()
    for i in range(10):
        for x, st, w, o in zip(b, streams, ws, outs):
            binding.attention_paged(x.site.cache, x.q, *x.pools, x.table_dev, x.lens_dev, o[i], x.qk_scale, workspace=w, stream=st)
    torch.cuda.synchronize()
    for o, w in zip(outs, want):
        assert all(torch.equal(t, w) for t in o)


def test_beside_the_contiguous_cache():
    """Code rows that a projection's epilogue wrote go into pages; the rows read back feed rptq_attention_kv, whose one-query
    output the paged call gives too (both are within their bounds of the same sums: half a step of the result each, and 2^-10 of the values)."""
    import torch
    from paper_2304_01089_b200 import binding
    from test_attention_gpu import Case
    H, d, T = 3, 128, 300
    c = Case(77, H=H, hd=d, gh=4, Tq=1, Tk=T)
    cache = binding.KvCache(c.LK, c.LV, H, 32)
    pools = [torch.zeros((12, n), dtype=torch.uint8, device="cuda") for n in (cache.k_page_bytes, cache.v_page_bytes)]
    pages = np.random.default_rng(1).permutation(12)[:10].astype(np.int32)
    slots = _slots(pages[np.arange(T) // 32].astype(np.int64) * 32 + np.arange(T) % 32)
    binding.kv_cache_write(cache, c.dk, c.dv, slots, *pools)
    back = [torch.zeros_like(c.dk), torch.zeros_like(c.dv)]
    binding.kv_cache_read(cache, *pools, slots, *back)
    assert torch.equal(back[0], c.dk) and torch.equal(back[1], c.dv)
    q = torch.randn((1, H * d), device="cuda").half()
    one, other = torch.empty_like(q), torch.empty_like(q)
    binding.attention_kv(c.LK, c.LV, H, q, back[0], back[1], one, c.qk_scale, True)
    binding.attention_paged(cache, q, *pools, torch.from_numpy(pages[None]).cuda(), torch.tensor([T], dtype=torch.int32, device="cuda"), other, c.qk_scale)
    top = float(c.sV.max()) * 15
    assert float((one.double() - other.double()).abs().max()) <= 2.0 ** -10 * top + 2 * 2.0 ** -11 * float(one.abs().max())
    assert binding.get_device_status() == 0


def test_refusals_on_the_device():
    import torch
    from paper_2304_01089_b200 import binding
    b = Batch(640, 2, 64, (4, 4), 16, [20])
    out = torch.empty_like(b.q)
    with pytest.raises(ValueError):                                          # fp32 queries have no kernel of the two types
        binding.attention_paged(b.site.cache, b.q, *b.pools, b.table_dev, b.lens_dev, out.float(), b.qk_scale)
    with pytest.raises(binding.RptqError) as e:
        binding.attention_paged(b.site.cache, b.q.float(), *b.pools, b.table_dev, b.lens_dev, out.float(), b.qk_scale)
    assert e.value.status == binding.ERR_INVALID_ARG
    with pytest.raises(ValueError):
        binding.attention_paged(b.site.cache, b.q, *b.pools, b.table_dev.long(), b.lens_dev, out, b.qk_scale)
    with pytest.raises(ValueError):
        binding.attention_paged(b.site.cache, b.q, *b.pools, b.table_dev, b.lens_dev, out, b.qk_scale, workspace=torch.empty(1, dtype=torch.uint8, device="cuda"))
    with pytest.raises(ValueError):
        binding.attention_paged(b.site.cache, b.q, b.pools[0], b.pools[1][:-1], b.table_dev, b.lens_dev, out, b.qk_scale)
    with pytest.raises(ValueError):
        binding.kv_cache_write(b.site.cache, b.q, b.q.float(), b.lens_dev.long(), *b.pools)
    with pytest.raises(ValueError):
        binding.kv_cache_write(b.site.cache, b.q, b.q, b.lens_dev, *b.pools)
    with pytest.raises(ValueError):
        binding.kv_cache_write(b.site.cache, b.q, b.q.cpu(), b.lens_dev.long(), *b.pools)
    # nothing to do is no error
    none = torch.empty((0, 128), dtype=torch.float16, device="cuda")
    binding.kv_cache_write(b.site.cache, none, none, torch.empty(0, dtype=torch.int64, device="cuda"), *b.pools)
    binding.kv_cache_read(b.site.cache, *b.pools, torch.empty(0, dtype=torch.int64, device="cuda"), none, none)
    binding.attention_paged(b.site.cache, none, *b.pools, b.table_dev[:0], b.lens_dev[:0], none, b.qk_scale)
    assert binding.get_device_status() == 0
