"""Shared by the tests of the paged key / value cache: sites, pools, and the definitions in 64 bits (numpy)."""
from __future__ import annotations

import numpy as np

HALF_STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8, "f32": 2.0 ** -24}
# Relative to a number of at least this size; below it the steps stay as they are at it (fp16: 2^-24 apart, so a rounding is off by up to 2^-25)
SMALLEST_NORMAL = {"f16": 2.0 ** -14, "bf16": 2.0 ** -126, "f32": 2.0 ** -126}


def torch_dtype(name):
    import torch
    return {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}[name]


class Tensor:
    """One tensor of the cache (K or V): a random reorder index with random cluster parameters, and its layout."""

    def __init__(self, rng, C, g, bits, order=0):
        from paper_2304_01089_b200 import binding
        self.bits, self.C = bits, C
        self.perm = rng.permutation(C).astype(np.int32)
        self.size = np.diff(np.concatenate([[0], np.sort(rng.integers(0, C + 1, size=g - 1)), [C]])).astype(np.int32)
        self.scale = rng.uniform(0.05, 0.4, size=g).astype(np.float32)
        self.zero = rng.integers(-2, (1 << bits) + 2, size=g).astype(np.int32)
        self.layout = binding.Layout(self.perm, self.size, self.scale, self.zero, bits, order=order)
        owner = np.empty(C, np.int64)
        owner[self.perm] = np.repeat(np.arange(g), self.size)
        self.s, self.z = self.scale[owner], self.zero[owner].astype(np.int64)      # of each channel

    def codes(self, x):
        """Eq. 1 in 64 bits: the exact product with the 32-bit reciprocal, rounded once, half to even."""
        inv = (1.0 / self.s.astype(np.float64)).astype(np.float32).astype(np.float64)
        t = np.rint(np.asarray(x, np.float64) * inv) + self.z
        return np.clip(np.nan_to_num(t, nan=-1e9, posinf=1e9, neginf=-1e9), 0, (1 << self.bits) - 1).astype(np.int64)

    def values(self, q):
        return self.s.astype(np.float64) * (q - self.z)

    def code_rows(self, q):
        """[n][C] codes -> [n][K_pad] in the padded order of the layout, pads 0."""
        idx = self.layout.padded_index()
        out = np.zeros((q.shape[0], idx.shape[0]), np.uint8)
        out[:, idx >= 0] = q[:, idx[idx >= 0]]
        return out

    def channels(self, rows):
        """The inverse of code_rows."""
        idx = self.layout.padded_index()
        out = np.zeros((rows.shape[0], self.C), np.int64)
        out[:, idx[idx >= 0]] = rows[:, idx >= 0]
        return out


class Site:
    def __init__(self, seed, H, d, bits, page, g=5, order=0):
        from paper_2304_01089_b200 import binding
        rng = np.random.default_rng(seed)
        self.H, self.d, self.C, self.page, self.rng = H, d, H * d, page, rng
        self.k, self.v = Tensor(rng, H * d, g, bits[0], order), Tensor(rng, H * d, g, bits[1], order)
        self.cache = binding.KvCache(self.k.layout, self.v.layout, H, page)

    def pools(self, n_pages, fill=0):
        import torch
        return [torch.full((n_pages, b), fill, dtype=torch.uint8, device="cuda") for b in (self.cache.k_page_bytes, self.cache.v_page_bytes)]

    def rows(self, n, dtype="f16", scale=1.0):
        """Rows of K and V on the device, and the same numbers in 64 bits."""
        import torch
        dev = [torch.from_numpy((self.rng.normal(size=(n, self.C)) * scale).astype(np.float32)).to(torch_dtype(dtype)).cuda() for _ in range(2)]
        return dev, [t.double().cpu().numpy() for t in dev]

    def read_codes(self, pools, slots):
        """The codes of these slots, through rptq_kv_cache_read and the host reader of packed rows."""
        import torch
        from paper_2304_01089_b200 import binding
        n = len(slots)
        out = [torch.zeros((n, t.layout.row_bytes), dtype=torch.uint8, device="cuda") for t in (self.k, self.v)]
        binding.kv_cache_read(self.cache, *pools, torch.from_numpy(np.asarray(slots, np.int64)).cuda(), *out)
        rows = [binding.codes_unpack_host(o.cpu().numpy(), t.layout.K_pad, t.bits) for o, t in zip(out, (self.k, self.v))]
        for r, t in zip(rows, (self.k, self.v)):
            assert not r[:, t.layout.padded_index() < 0].any()
        return [t.channels(r) for r, t in zip(rows, (self.k, self.v))]


class Batch:
    """Sequences of the given lengths in shuffled pages of a pool, with random rows written."""

    def __init__(self, seed, H, d, bits, page, lens, G=1, dtype="f16", fill=0, q_scale=1.0, spare=2, g=5):
        import torch
        from paper_2304_01089_b200 import binding
        self.site = s = Site(seed, H, d, bits, page, g=g)
        self.lens, self.G, self.dtype = list(lens), G, dtype
        need = [-(-n // page) for n in lens]
        self.n_pages = sum(need) + spare
        self.width = max(1, max(need, default=1))
        ids = s.rng.permutation(self.n_pages)[:sum(need)].astype(np.int32)
        self.table = np.full((len(lens), self.width), -1, np.int32)
        self.table[np.arange(self.width)[None, :] < np.array(need, int).reshape(-1, 1)] = ids
        at = [self.table[i, np.arange(n) // page].astype(np.int64) * page + np.arange(n) % page for i, n in enumerate(lens)]
        self.slots = np.concatenate(at) if at else np.zeros(0, np.int64)
        self.pools = s.pools(self.n_pages, fill)
        dev, x = s.rows(len(self.slots), dtype)
        binding.kv_cache_write(s.cache, *dev, torch.from_numpy(self.slots).cuda(), *self.pools)
        self.kq, self.vq = s.k.codes(x[0]), s.v.codes(x[1])
        self.qk_scale = 1.0 / np.sqrt(d)
        self.q = torch.from_numpy((s.rng.normal(size=(len(lens), H * G * d)) * q_scale).astype(np.float32)).to(torch_dtype(dtype)).cuda()
        self.table_dev, self.lens_dev = torch.from_numpy(self.table).cuda(), torch.tensor(self.lens, dtype=torch.int32, device="cuda")

    def run(self, **kw):
        import torch
        from paper_2304_01089_b200 import binding
        out = torch.full_like(self.q, float("nan"))
        binding.attention_paged(self.site.cache, self.q, *self.pools, self.table_dev, self.lens_dev, out, self.qk_scale,
                                n_q_heads=self.site.H * self.G, **kw)
        torch.cuda.synchronize()
        return out

    def want(self):
        """([n_seq][H * G * d] outputs in 64 bits, what a kernel may be off).

        A score is a sum of d products in at least 32 bits, each of a query times a scale (one rounding) with a code, times one
        factor: with A = qk_scale log2(e) sum |q s| (2^bits - 1) its error is at most (d + 8) 2^-24 A in units of the exponent of 2, so a
        probability is off by a factor of 1 +- E, E = (d + 8) 2^-24 A + 2^-20 (the second term: ex2 and the rounding of its argument), or
        by 2^-25 of the largest where it is held as an integer. Probabilities in numerator and denominator give twice that; the sums
        over n keys in 32 bits add (n + 8) 2^-24 in the worst case, where fp16 pairs carry the probabilities another 2^-20. The
        result is rounded once to the output's type."""
        s, d, G = self.site, self.site.d, self.G
        q = self.q.double().cpu().numpy().reshape(len(self.lens), s.H, G, d)
        out, bound = np.zeros_like(q), np.zeros_like(q)
        at = 0
        for i, n in enumerate(self.lens):
            if n == 0:
                continue
            kq, vq = self.kq[at:at + n], self.vq[at:at + n]
            at += n
            K, V = s.k.values(kq).reshape(n, s.H, d), s.v.values(vq).reshape(n, s.H, d)
            S = self.qk_scale * np.einsum("hgd,nhd->hgn", q[i], K)
            top = S.max(-1, keepdims=True)
            P = np.exp(S - top)
            total = P.sum(-1, keepdims=True)
            P /= total
            out[i] = np.einsum("hgn,nhd->hgd", P, V)
            A = self.qk_scale * 1.4427 * np.abs(q[i] * s.k.s.astype(np.float64).reshape(s.H, 1, d)).sum(-1, keepdims=True) * ((1 << s.k.bits) - 1)
            E = (d + 8) * 2.0 ** -24 * A + 2.0 ** -19
            reach = np.abs(s.v.s.astype(np.float64)).reshape(1, s.H, d) * np.maximum(vq, np.abs(vq - s.v.z)).reshape(n, s.H, d)   # codes and values
            mass = np.einsum("hgn,nhd->hgd", P + 2.0 ** -25 / total, reach)
            bound[i] = (2 * E + (n + 8) * 2.0 ** -24) * mass + 2 * n * 2.0 ** -25 / total * reach.max(0)[:, None, :] + 1e-30
        bound += HALF_STEP[self.dtype] * np.maximum(np.abs(out) + bound, SMALLEST_NORMAL[self.dtype])
        return out.reshape(len(self.lens), -1), bound.reshape(len(self.lens), -1)

    def check(self, **kw):
        out = self.run(**kw)
        got = out.double().cpu().numpy()
        want, bound = self.want()
        assert np.isfinite(got).all()
        off = np.abs(got - want) - bound
        assert (off <= 0).all(), (float(off.max()), float(np.abs(got - want).max()), np.unravel_index(off.argmax(), off.shape))
        for i, n in enumerate(self.lens):
            if n == 0:
                assert not got[i].any()
        return out
