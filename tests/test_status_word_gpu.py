"""The device's status word: what a call records does not hide what an earlier one recorded."""
import numpy as np
import pytest

from paged_cases import Batch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("call", ["write", "write codes", "read", "read codes", "attend"])
def test_a_slot_outside_the_pool_does_not_hide_a_wait_that_ran_out(call):
    """A wait that ran out leaves an output undefined, a bad slot or page only leaves something out."""
    import torch
    from paper_2304_01089_b200 import binding
    b = Batch(720, 2, 64, (4, 4), 16, [40, 20])
    past = torch.tensor([b.n_pages * 16, -1], device="cuda")
    codes = [torch.zeros((2, t.layout.row_bytes), dtype=torch.uint8, device="cuda") for t in (b.site.k, b.site.v)]
    x = torch.zeros((2, 128), dtype=torch.float16, device="cuda")
    b.table_dev[0, 1] = b.n_pages

    def bad():
        if call == "attend":
            b.run()
        elif call.startswith("write"):
            binding.kv_cache_write(b.site.cache, *(codes if "codes" in call else (x, x.clone())), past, *b.pools)
        else:
            binding.kv_cache_read(b.site.cache, *b.pools, past, *(codes if "codes" in call else (x, x.clone())))

    L = binding.Layout(np.arange(64), [64], [0.1], [3], 4)
    ones, rows = torch.ones(64, dtype=torch.float16, device="cuda"), torch.zeros((600, 64), dtype=torch.float16, device="cuda")
    out = torch.zeros((600, L.row_bytes), dtype=torch.uint8, device="cuda")
    ran_out = lambda: binding.selftest_ln_timeout(L, rows, ones, ones, 1e-5, out)
    assert binding.get_device_status() == 0
    for calls, status in (((bad,), binding.ERR_BAD_SLOT), ((ran_out, bad), binding.ERR_DEVICE_TIMEOUT), ((bad, ran_out), binding.ERR_DEVICE_TIMEOUT)):
        for f in calls:
            f()
        assert binding.get_device_status() == status
        assert binding.get_device_status() == 0
