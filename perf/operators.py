"""The paged, quantised key / value cache, as cases that can be timed and compared.

A case is one pass of a serving program over data that is on the device already. Kinds ("op"):

  attend  one new token per sequence attends over the sequence's pages          (binding.attention_paged)
  append  the keys and values of new tokens are quantised into their pages, and
          rows of the cache are read back as the values that the codes stand for (binding.kv_cache_write, kv_cache_read)
  read    rows of the cache are read back                                       (binding.kv_cache_read)

The plain forms keep one byte per code, [slots][heads][head_dim], and work in 32 bits; the framework keeps its packed pages.
Both start from the same keys, values, parameters and page tables.

Each cached head has four clusters of channels (by the channels' ranges) with one scale and zero point each, from the ranges of a
calibration sample, as the attention sites of the paper do. The sequences of a case have lengths between nothing (a padded row of the
batch) and "tokens"; they follow from the case alone, so that a case's shapes and work do not depend on the seed.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

CLUSTERS = 4                     # per head
CALIBRATION_TOKENS = 256
DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
# what a drawn case may cost: no more than the largest listed ones
MAX_CACHED = 2.7e8               # seqs x tokens x heads x head_dim, the plain form's dense cache
MAX_ROWS = 3.7e7                 # rows x heads x head_dim that are read back as values


def listed():
    return [
        # one user of the smallest model, a short conversation: launches and latency
        dict(name="attend 1x100 12h64 4b", op="attend", seqs=1, tokens=100, heads=12, group=1, head_dim=64, bits_k=4, bits_v=4, dtype="f16", page=16),
        # a decode step of the benchmark's heads for eight users of ragged lengths
        dict(name="attend 8x2011 72h128 4b", op="attend", seqs=8, tokens=2011, heads=72, group=1, head_dim=128, bits_k=4, bits_v=4, dtype="f16", page=16),
        # one user with a very long context: the length has to be split
        dict(name="attend 1x65553 32h128 4b", op="attend", seqs=1, tokens=65553, heads=32, group=1, head_dim=128, bits_k=4, bits_v=4, dtype="bf16", page=64),
        # a large batch of short contexts, four query heads on each cached head, 8-bit cache
        dict(name="attend 64x1337 8x4h128 8b", op="attend", seqs=64, tokens=1337, heads=8, group=4, head_dim=128, bits_k=8, bits_v=8, dtype="bf16", page=32),
        # the largest model's heads with the paper's 3-bit cache
        dict(name="attend 16x1700 96h128 3b", op="attend", seqs=16, tokens=1700, heads=96, group=1, head_dim=128, bits_k=3, bits_v=3, dtype="f16", page=16),
        # odd sizes: heads of 80 channels, keys and values of different bits, pages that are no power of two, eight query heads a cached head
        dict(name="attend 5x333 4x8h80 k4v8", op="attend", seqs=5, tokens=333, heads=4, group=8, head_dim=80, bits_k=4, bits_v=8, dtype="f16", page=48),
        # a decode step writes one token for each of eight users and takes back their last 16 rows
        dict(name="append 8x1 72h128 4b", op="append", seqs=8, tokens=2011, new=1, window=16, heads=72, head_dim=128, bits_k=4, bits_v=4, dtype="f16", page=16),
        # chunks of three prompts on what is cached of them; the chunk attends over all of it
        dict(name="append 3x333 32h64 8b", op="append", seqs=3, tokens=833, new=333, window=833, heads=32, head_dim=64, bits_k=8, bits_v=8, dtype="bf16", page=32),
        # the benchmark's whole prompt of 4096 tokens
        dict(name="append 1x4096 72h128 4b", op="append", seqs=1, tokens=4096, new=4096, window=4096, heads=72, head_dim=128, bits_k=4, bits_v=4, dtype="f16", page=16),
        # a few cached rows of a small model, to be looked at in fp32
        dict(name="read 1x37 12h64 4b", op="read", seqs=1, tokens=37, heads=12, head_dim=64, bits_k=4, bits_v=4, dtype="f32", page=16),
        # a cached prefix of the benchmark's model, for the next chunk of its prompt
        dict(name="read 1x2011 72h128 3b", op="read", seqs=1, tokens=2011, heads=72, head_dim=128, bits_k=3, bits_v=3, dtype="f16", page=16),
        # sixteen users' caches handed over to another worker
        dict(name="read 16x900 32h128 8b", op="read", seqs=16, tokens=900, heads=32, head_dim=128, bits_k=8, bits_v=8, dtype="bf16", page=128),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], spread over the logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "attend", "append", "append", "read"])
    bits_k = rng.choice([3, 4, 4, 8])
    case = dict(op=op, seqs=_log(rng, 1, 64), tokens=_log(rng, 1, 8000), heads=_log(rng, 2, 96), head_dim=rng.choice([64, 64, 80, 96, 128, 128, 128, 256]),
                bits_k=bits_k, bits_v=rng.choice([bits_k, bits_k, bits_k, 3, 4, 8]), page=rng.choice([16, 16, 32, 48, 64, 128, 256]))
    if op == "attend":
        case.update(group=rng.choice([1, 1, 1, 1, 2, 3, 4, 8]), dtype=rng.choice(["f16", "bf16"]))
        if rng.random() < 0.25:
            case.update(seqs=rng.randint(1, 2), tokens=_log(rng, 8000, 65000), heads=_log(rng, 2, 32))
    else:
        case.update(dtype=rng.choice(["f16", "f16", "bf16", "bf16", "f32"]))
    dense = lambda: case["seqs"] * case["tokens"] * case["heads"] * case["head_dim"]
    while dense() > (MAX_CACHED if op != "read" else MAX_ROWS):
        at = max(("seqs", "tokens", "heads"), key=lambda n: case[n])
        case[at] = max(1, case[at] * 2 // 3)
    if op == "append":
        case["new"] = rng.choice([1, case["tokens"], rng.randint(1, case["tokens"])])
        case["window"] = rng.choice([case["new"], case["tokens"]])
        while case["seqs"] * case["window"] * case["heads"] * case["head_dim"] > MAX_ROWS:
            case["window"] = max(1, case["window"] // 2)
            case["new"] = min(case["new"], case["window"])
    return case


def _lengths(case):
    """Tokens of each sequence, the new ones included: the first has them all, of the others one in sixteen is a padded row."""
    rng = random.Random("%d %d %d %d" % (case["seqs"], case["tokens"], case["heads"], case["page"]))
    new = case.get("new", 0)
    return [case["tokens"]] + [0 if rng.random() < 1 / 16 else rng.randint(max(1, new), case["tokens"]) for _ in range(case["seqs"] - 1)]


def work(case):
    lens, C, e = _lengths(case), case["heads"] * case["head_dim"], 4 if case["dtype"] == "f32" else 2
    bits = case["bits_k"] + case["bits_v"]
    total, new = sum(lens), sum(min(n, case.get("new", 0)) for n in lens)
    if case["op"] == "attend":
        q = case["seqs"] * C * case["group"]
        return {"bytes": total * C * bits / 8 + 2 * q * e + 4 * sum(-(-n // case["page"]) for n in lens) + 4 * case["seqs"],
                "flops": 4 * total * C * case["group"]}
    back = total if case["op"] == "read" else sum(min(n, case["window"]) for n in lens)
    return {"bytes": new * (2 * C * e + C * bits / 8 + 8) + back * (2 * C * e + C * bits / 8 + 8), "flops": 4 * (new + back) * C}


# ---------------------------------------------------------------- inputs
def _channels(gen, case):
    """What the rows of one tensor look like: each channel's spread and middle; one channel in a hundred is eight times larger."""
    C = case["heads"] * case["head_dim"]
    spread = torch.exp(0.4 * torch.randn(C, device="cuda", generator=gen))
    spread = torch.where(torch.rand(C, device="cuda", generator=gen) < 0.01, 8.0 * spread, spread)
    return spread, 0.5 * spread * torch.randn(C, device="cuda", generator=gen)


def _rows(gen, channels, n, dtype):
    spread, middle = channels
    return (torch.randn((n, spread.shape[0]), device="cuda", generator=gen) * spread + middle).to(dtype)


def _clusters(gen, case, channels, bits):
    """Each head's channels in the order of their calibrated ranges, cut into clusters; Min-Max parameters of each cluster (the
    paper's Eq. 2, codes counted from 0). Returns (perm, size, scale, zero) and each channel's scale and zero point."""
    H, d = case["heads"], case["head_dim"]
    sample = _rows(gen, channels, CALIBRATION_TOKENS, torch.float32)
    lo, hi = sample.amin(0).view(H, d), sample.amax(0).view(H, d)
    order = torch.argsort(hi - lo, dim=1)
    cut = [0, d // 3 + 1, d // 2 + 2, d - max(1, d // 16), d]            # many small ranges, few large ones
    size = [b - a for a, b in zip(cut, cut[1:])]
    owner = torch.repeat_interleave(torch.arange(CLUSTERS, device="cuda"), torch.tensor(size, device="cuda")).expand(H, d)
    low = torch.full((H, CLUSTERS), math.inf, device="cuda").scatter_reduce_(1, owner, lo.gather(1, order), "amin")
    high = torch.full((H, CLUSTERS), -math.inf, device="cuda").scatter_reduce_(1, owner, hi.gather(1, order), "amax")
    scale = (high - low) / (1 << bits)
    zero = (1 << (bits - 1)) - torch.round((high + low) / (2 * scale))
    of_channel = torch.empty_like(order).scatter_(1, order, owner)        # the cluster of each channel of each head
    perm = order + d * torch.arange(H, device="cuda")[:, None]
    return dict(perm=perm.flatten(), size=size * H, scale=scale.flatten(), zero=zero.flatten().to(torch.int32),
                channel_scale=scale.gather(1, of_channel).flatten(), channel_zero=zero.gather(1, of_channel).flatten())


def _inputs(case, seed):
    """Everything that a pass starts from, in no particular form of the cache: parameters, the rows that are cached already with
    their slots, the page table, the new rows or the query."""
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    lens, page, dtype = _lengths(case), case["page"], DTYPES[case["dtype"]]
    kc, vc = _channels(gen, case), _channels(gen, case)
    s = dict(case=case, lens=lens, k_par=_clusters(gen, case, kc, case["bits_k"]), v_par=_clusters(gen, case, vc, case["bits_v"]))
    pages = [-(-n // page) for n in lens]
    width = max(1, max(pages))
    s["n_pages"] = sum(pages) + 3 + sum(pages) // 16                     # the pool is larger than what is in use
    pool = torch.randperm(s["n_pages"], device="cuda", generator=gen)[:sum(pages)].cpu().numpy()
    table = np.full((len(lens), width), -1, np.int32)
    table[np.arange(width)[None, :] < np.array(pages)[:, None]] = pool
    s["table"] = torch.from_numpy(table).cuda()
    s["seq_lens"] = torch.tensor(lens, dtype=torch.int32, device="cuda")

    def slots(first, last):
        """Slots of the tokens first[i] .. last[i] - 1 of each sequence, one sequence after the other."""
        at = [(table[i, np.arange(a, b) // page].astype(np.int64) * page + np.arange(a, b) % page) for i, (a, b) in enumerate(zip(first, last))]
        return torch.from_numpy(np.concatenate(at)).cuda()

    new = case.get("new", 0)
    old = [max(0, n - new) for n in lens]
    s["old_slots"] = slots([0] * len(lens), old)
    s["old_k"], s["old_v"] = _rows(gen, kc, sum(old), dtype), _rows(gen, vc, sum(old), dtype)
    if case["op"] == "attend":
        s["q"] = torch.randn((case["seqs"], case["heads"] * case["group"] * case["head_dim"]), device="cuda", generator=gen).to(dtype)
        s["qk_scale"] = 1.0 / math.sqrt(case["head_dim"])
        return s
    if case["op"] == "append":
        s["new_slots"] = slots(old, lens)
        s["new_k"], s["new_v"] = _rows(gen, kc, sum(lens) - sum(old), dtype), _rows(gen, vc, sum(lens) - sum(old), dtype)
    s["read_slots"] = slots([max(0, n - case.get("window", n)) for n in lens], lens)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    rows, dtype, C = case["page"] * s["n_pages"], DTYPES[case["dtype"]], case["heads"] * case["head_dim"]
    if own:
        from paper_2304_01089_b200 import binding
        host = lambda t: t.cpu().numpy()
        lay = [binding.Layout(host(p["perm"]), p["size"], host(p["scale"]), host(p["zero"]), bits)
               for p, bits in ((s["k_par"], case["bits_k"]), (s["v_par"], case["bits_v"]))]
        s["cache"] = c = binding.KvCache(lay[0], lay[1], case["heads"], case["page"])
        s["k_pages"] = torch.zeros((s["n_pages"], c.k_page_bytes), dtype=torch.uint8, device="cuda")
        s["v_pages"] = torch.zeros((s["n_pages"], c.v_page_bytes), dtype=torch.uint8, device="cuda")
        binding.kv_cache_write(c, s["old_k"], s["old_v"], s["old_slots"], s["k_pages"], s["v_pages"])
        if case["op"] == "attend":
            s["out"] = torch.empty_like(s["q"])
            s["workspace"] = torch.empty(binding.attention_paged_workspace_bytes(c, case["heads"] * case["group"]), dtype=torch.uint8, device="cuda")
        else:
            s["k_out"], s["v_out"] = (torch.empty((s["read_slots"].shape[0], C), dtype=dtype, device="cuda") for _ in range(2))
    else:
        s["k_codes"], s["v_codes"] = (torch.zeros((rows, C), dtype=torch.uint8, device="cuda") for _ in range(2))
        _write(s, "old")
    del s["old_k"], s["old_v"]
    return s


# ---------------------------------------------------------------- the plain forms
def _quantise(x, par, bits):
    """Codes of rows: the product with the 32-bit reciprocal of the scale in 64 bits (exact), rounded once, half to even."""
    inv = (1.0 / par["channel_scale"].double()).float().double()
    return (torch.round(x.double() * inv) + par["channel_zero"].double()).clamp_(0, (1 << bits) - 1).to(torch.uint8)


def _values(codes, par):
    return (codes.float() - par["channel_zero"]) * par["channel_scale"]


def _write(s, which):
    case, at = s["case"], s[which + "_slots"]
    s["k_codes"][at] = _quantise(s[which + "_k"], s["k_par"], case["bits_k"])
    s["v_codes"][at] = _quantise(s[which + "_v"], s["v_par"], case["bits_v"])


def _read(s):
    dtype = DTYPES[s["case"]["dtype"]]
    return _values(s["k_codes"][s["read_slots"]], s["k_par"]).to(dtype), _values(s["v_codes"][s["read_slots"]], s["v_par"]).to(dtype)


def _attend(s):
    case, table = s["case"], s["table"]
    B, H, G, d, page = case["seqs"], case["heads"], case["group"], case["head_dim"], case["page"]
    key = torch.arange(max(1, case["tokens"]), device="cuda")
    slot = table[:, key // page].clamp(min=0).long() * page + key % page                       # [B][L]
    seen = key[None, :] < s["seq_lens"][:, None]
    q = s["q"].float().view(B, H, G, d)
    k = _values(s["k_codes"][slot], s["k_par"]).view(B, -1, H, d).permute(0, 2, 3, 1)          # [B][H][d][L]
    score = (q @ k) * s["qk_scale"]
    score = score.masked_fill(~seen[:, None, None, :], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = torch.exp(score - torch.where(torch.isinf(top), torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    v = _values(s["v_codes"][slot], s["v_par"]).view(B, -1, H, d).permute(0, 2, 1, 3)          # [B][H][L][d]
    out = (p @ v) / torch.where(total > 0, total, torch.ones_like(total))
    return out.reshape(B, H * G * d).to(s["q"].dtype)


# ---------------------------------------------------------------- one pass
def run(state):
    case = state["case"]
    if own:
        from paper_2304_01089_b200 import binding
        if case["op"] == "attend":
            binding.attention_paged(state["cache"], state["q"], state["k_pages"], state["v_pages"], state["table"], state["seq_lens"], state["out"],
                                    state["qk_scale"], n_q_heads=case["heads"] * case["group"], workspace=state["workspace"])
            return state["out"]
        if case["op"] == "append":
            binding.kv_cache_write(state["cache"], state["new_k"], state["new_v"], state["new_slots"], state["k_pages"], state["v_pages"])
        binding.kv_cache_read(state["cache"], state["k_pages"], state["v_pages"], state["read_slots"], state["k_out"], state["v_out"])
        return state["k_out"], state["v_out"]
    if case["op"] == "attend":
        return _attend(state)
    if case["op"] == "append":
        _write(state, "new")
    return _read(state)


# ---------------------------------------------------------------- the definition in 64 bits
def exact(case, seed):
    s = _inputs(case, seed)
    H, G, d, page = case["heads"], case.get("group", 1), case["head_dim"], case["page"]
    dev = "cuda"

    def cached(par, bits, rows):
        """The values that the codes of these rows stand for."""
        scale = par["channel_scale"].to(torch.float64)
        zero = par["channel_zero"].to(torch.float64)
        steps = rows.to(torch.float64) * torch.reciprocal(scale).to(torch.float32).to(torch.float64)
        low, high = -zero, (1 << bits) - 1 - zero                        # the codes' ends, counted from the zero point
        return scale * torch.minimum(torch.maximum(torch.round(steps), low), high)

    if case["op"] != "attend":
        # where each slot's row is: among the old rows, then the new ones
        k, v = s["old_k"], s["old_v"]
        place = torch.full((page * s["n_pages"],), -1, dtype=torch.int64, device=dev)
        place[s["old_slots"]] = torch.arange(k.shape[0], device=dev)
        if case["op"] == "append":
            place[s["new_slots"]] = k.shape[0] + torch.arange(s["new_k"].shape[0], device=dev)
            k, v = torch.cat([k, s["new_k"]]), torch.cat([v, s["new_v"]])
        take = place[s["read_slots"]]
        return cached(s["k_par"], case["bits_k"], k[take]), cached(s["v_par"], case["bits_v"], v[take])
    out = torch.zeros((case["seqs"], H * G, d), dtype=torch.float64, device=dev)
    at = 0
    for i, n in enumerate(s["lens"]):
        if n == 0:
            continue
        q = s["q"][i].to(torch.float64).view(H, G, d)
        k = cached(s["k_par"], case["bits_k"], s["old_k"][at:at + n]).view(n, H, d)
        weight = torch.softmax(s["qk_scale"] * torch.einsum("hgd,nhd->hgn", q, k), dim=-1)
        v = cached(s["v_par"], case["bits_v"], s["old_v"][at:at + n]).view(n, H, d)
        out[i] = torch.einsum("hgn,nhd->hgd", weight, v).reshape(H * G, d)
        at += n
    return out.reshape(case["seqs"], H * G * d)
