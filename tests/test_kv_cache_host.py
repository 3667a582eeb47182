"""The paged cache's boundary without a device: sizes, and every refusal of a call, which comes before any launch."""
import ctypes as C

import numpy as np
import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_2304_01089_b200 import build as lib_build
    lib_build.build()
    from paper_2304_01089_b200 import binding as b
    return b


def _layout(b, channels, bits):
    return b.Layout(np.arange(channels), [channels], [0.5], [3], bits)


def test_page_sizes(binding):
    for H, d, page, bk, bv in [(2, 64, 16, 3, 4), (12, 64, 32, 4, 8), (3, 40, 48, 8, 3), (1, 256, 65536, 4, 4)]:
        c = binding.KvCache(_layout(binding, H * d, bk), _layout(binding, H * d, bv), H, page)
        dp = (d + 31) // 32 * 32
        assert (c.k_page_bytes, c.v_page_bytes) == (page * H * dp * bk // 8, page * H * dp * bv // 8)
        assert c.k_page_bytes % 16 == 0 and c.v_page_bytes % 16 == 0
        c.destroy()
        with pytest.raises(ValueError):
            c.handle


def test_create_refuses(binding):
    L, M = _layout(binding, 128, 4), _layout(binding, 64, 4)
    for args, status in [((L, M, 2, 16), binding.ERR_INVALID_ARG), ((L, L, 3, 16), binding.ERR_INVALID_ARG), ((L, L, 0, 16), binding.ERR_INVALID_ARG),
                         ((L, L, 2, 0), binding.ERR_INVALID_ARG), ((L, L, 2, 24), binding.ERR_UNSUPPORTED), ((L, L, 2, 65552), binding.ERR_UNSUPPORTED),
                         ((_layout(binding, 512, 4), _layout(binding, 512, 4), 1, 16), binding.ERR_UNSUPPORTED)]:
        with pytest.raises(binding.RptqError) as e:
            binding.KvCache(*args)
        assert e.value.status == status
    lib = binding._lib
    assert lib.rptq_kv_cache_create(None, L.handle, L.handle, 2, 16) == binding.ERR_INVALID_ARG
    h = C.c_void_p(1)
    assert lib.rptq_kv_cache_create(C.byref(h), None, L.handle, 2, 16) == binding.ERR_INVALID_ARG and not h.value
    assert lib.rptq_kv_cache_query(None, None, None) == binding.ERR_INVALID_ARG
    assert lib.rptq_kv_cache_destroy(None) == binding.OK
    assert binding.status_string(binding.ERR_BAD_SLOT) == "slot or page outside its pool"


# Addresses that nothing reads: a refused call returns before it looks at them, and without a device no call gets further.
A, ODD = 1 << 20, (1 << 20) + 1


def test_write_and_read_refuse(binding):
    import torch
    cache = binding.KvCache(_layout(binding, 128, 4), _layout(binding, 128, 4), 2, 16)
    lib, inv = binding._lib, binding.ERR_INVALID_ARG
    rb = cache.k_row_bytes
    good = dict(k=A, ldk=128, v=A, ldv=128, kind=binding.ROWS_F16, slots=A, n=4, kp=A, vp=A, pages=3)

    def write(**kw):
        g = dict(good, **kw)
        return lib.rptq_kv_cache_write(g.get("cache", cache.handle), g["k"], g["ldk"], g["v"], g["ldv"], g["kind"], g["slots"], g["n"], g["kp"], g["vp"], g["pages"], None)

    def read(**kw):
        g = dict(good, **kw)
        return lib.rptq_kv_cache_read(g.get("cache", cache.handle), g["kp"], g["vp"], g["pages"], g["slots"], g["n"], g["k"], g["ldk"], g["v"], g["ldv"], g["kind"], None)

    bad = [dict(cache=None), dict(k=None), dict(v=None), dict(slots=None), dict(kp=None), dict(vp=None), dict(n=-1), dict(pages=-1), dict(ldk=127), dict(ldv=127),
           dict(kind=4), dict(kind=-1), dict(k=ODD), dict(v=ODD), dict(kp=A + 8), dict(vp=A + 8), dict(slots=A + 4), dict(kind=binding.ROWS_F32, k=A + 2),
           dict(kind=binding.ROWS_CODES, ldk=rb - 4, ldv=rb), dict(kind=binding.ROWS_CODES, ldk=rb + 2, ldv=rb), dict(kind=binding.ROWS_CODES, ldk=rb, ldv=rb, k=A + 2)]
    for kw in bad:
        assert write(**kw) == inv and read(**kw) == inv, kw
    assert write(pages=1 << 60) == binding.ERR_UNSUPPORTED
    assert write(n=0) == binding.OK and read(n=0, k=None, v=None, slots=None) == binding.OK
    if not torch.cuda.is_available():
        assert write() == binding.ERR_CUDA and read() == binding.ERR_CUDA      # the arguments are right, a device is missing


def test_attention_refuses(binding):
    import torch
    cache = binding.KvCache(_layout(binding, 128, 4), _layout(binding, 128, 4), 2, 16)
    lib, inv, uns = binding._lib, binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    good = dict(q=A, ldq=256, kind=binding.ROWS_F16, heads=4, seqs=3, kp=A, vp=A, pages=9, table=A, ldt=5, width=5, lens=A, scale=0.1, out=A, ldo=256, ws=A)

    def call(**kw):
        g = dict(good, **kw)
        return lib.rptq_attention_paged(g.get("cache", cache.handle), g["q"], g["ldq"], g["kind"], g["heads"], g["seqs"], g["kp"], g["vp"], g["pages"], g["table"],
                                        g["ldt"], g["width"], g["lens"], C.c_float(g["scale"]), g["out"], g["ldo"], g["ws"], None)

    for kw in [dict(cache=None), dict(q=None), dict(out=None), dict(kp=None), dict(vp=None), dict(table=None), dict(lens=None), dict(ws=None), dict(seqs=-1), dict(pages=-1),
               dict(width=-1), dict(ldt=4), dict(heads=0), dict(heads=3), dict(ldq=255), dict(ldo=255), dict(kind=binding.ROWS_F32), dict(kind=binding.ROWS_CODES),
               dict(q=ODD), dict(out=ODD), dict(kp=A + 4), dict(vp=A + 4), dict(table=A + 2), dict(lens=A + 2), dict(ws=A + 8), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))]:
        assert call(**kw) == inv, kw
    assert call(seqs=65536) == uns and call(width=1 << 28, ldt=1 << 28) == uns
    assert call(seqs=60000, width=1 << 16, ldt=1 << 16) == uns             # more tiles than the list has places
    assert call(seqs=0, q=None) == binding.OK
    if not torch.cuda.is_available():
        assert call() == binding.ERR_CUDA
    assert lib.rptq_attention_paged_workspace_bytes(None, 2) == inv
    assert lib.rptq_attention_paged_workspace_bytes(cache.handle, 3) == inv
    with pytest.raises(binding.RptqError):
        binding.attention_paged_workspace_bytes(cache, 5)


def test_tensors_that_do_not_fit_are_refused(binding):
    """The marshalling in front of the library, on CPU tensors where there is no device (with one they are on the wrong device)."""
    import torch
    cache = binding.KvCache(_layout(binding, 128, 4), _layout(binding, 128, 3), 2, 16)
    pools = [torch.zeros((3, b), dtype=torch.uint8) for b in (cache.k_page_bytes, cache.v_page_bytes)]
    k, slots = torch.zeros((5, 130)), torch.zeros(5, dtype=torch.int64)
    codes = [torch.zeros((5, b), dtype=torch.uint8) for b in (cache.k_row_bytes, cache.v_row_bytes)]
    q, out = torch.zeros((4, 256), dtype=torch.float16), torch.zeros((4, 260), dtype=torch.float16)
    table, lens, ws = torch.zeros((4, 2), dtype=torch.int32), torch.zeros(4, dtype=torch.int32), torch.zeros(64, dtype=torch.uint8)
    cache._workspace[4] = 64                                                # (its size is the device's to say)
    write = lambda *a, **kw: binding.kv_cache_write(cache, *a, **kw)
    read = lambda *a, **kw: binding.kv_cache_read(cache, *a, **kw)
    attend = lambda *a, **kw: binding.attention_paged(cache, *a, 0.1, n_q_heads=4, workspace=kw.pop("workspace", ws), **kw)
    if not torch.cuda.is_available():
        for call in (lambda: write(k, k, slots, *pools), lambda: write(k[:, 2:], k[:, 1:129], slots, *pools), lambda: write(*codes, slots, *pools),
                     lambda: read(*pools, slots, k, k), lambda: read(*pools, slots[:2], *codes), lambda: attend(q, *pools, table, lens, out),
                     lambda: attend(q[:1], *pools, table[:1, :1], lens[:1], out[:1, 4:])):
            with pytest.raises(binding.RptqError) as e:                       # all arguments pass, a device is missing
                call()
            assert e.value.status == binding.ERR_CUDA
    for call in (lambda: write(k, k, slots.int(), *pools), lambda: write(k, k, slots[::2], *pools), lambda: write(k[:4], k, slots, *pools),
                 lambda: write(k[:, 3:], k, slots, *pools), lambda: write(k, k.half(), slots, *pools), lambda: write(k.double(), k.double(), slots, *pools),
                 lambda: write(k.t(), k, slots, *pools), lambda: write(k[0], k[0], slots, *pools), lambda: write(codes[1], codes[0][:, 1:], slots, *pools),
                 lambda: write(k, k, slots, pools[0], pools[1][:2]), lambda: write(k, k, slots, pools[1], pools[0]), lambda: write(k, None, slots, *pools),
                 lambda: write(k, k, slots, pools[0].to(torch.int8), pools[1]), lambda: read(pools[0][:, ::2], pools[1], slots, k, k),
                 lambda: read(*pools, slots, k[:, ::2], k), lambda: attend(q, *pools, table.long(), lens, out), lambda: attend(q, *pools, table, lens.long(), out),
                 lambda: attend(q, *pools, table[:3], lens, out), lambda: attend(q, *pools, table, lens, out.float()), lambda: attend(q[:3], *pools, table, lens, out),
                 lambda: attend(q[:, 1:], *pools, table, lens, out), lambda: attend(q, *pools, table, lens[None], out), lambda: attend(q, *pools, table[:, 0], lens, out),
                 lambda: attend(q, *pools, table, lens, out, workspace=ws[:60]), lambda: attend(q, *pools, table, lens, out, workspace=ws.repeat(2)[::2])):
        with pytest.raises(ValueError):
            call()
    cache.destroy()
    with pytest.raises(ValueError):
        write(k, k, slots, *pools)
    with pytest.raises(ValueError):
        attend(q, *pools, table, lens, out)
