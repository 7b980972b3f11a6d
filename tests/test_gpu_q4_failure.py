"""Bounded waits of the tile kernel over a cache of 4 bits: a limit that runs out is reported, every role leaves, no copy is
on its way when a block does, and the context serves the next call.  The kernel for few rows waits for nothing."""
import pytest
import torch

import paper_2508_02401_gb300 as ckv
from tests import attention_ref as ref
from tests.test_gpu_attention_failure import _built, calls_after_calls_that_gave_up, one_microsecond  # noqa: F401
from tests.test_gpu_prefill_attention import config
from tests.test_gpu_q4_attention import Paged4

pytestmark = pytest.mark.gpu


def arguments(c):
    return [torch.as_tensor(x, dtype=torch.int32, device="cuda") for x in (c.table, c.lens, c.cu)]


@pytest.mark.parametrize("new", [9, 20, 70])
def test_chunks(one_microsecond, new):  # noqa: F811
    c = Paged4(config(), (3000, 700, 90), (new,) * 3, 32, seed=21)
    ws, cache, out = ckv.new_attention_workspace(c.cfg), ckv.PagedCacheQ4(c.pages, 32), torch.zeros_like(c.q)
    table, lens, cu = arguments(c)
    for _ in range(3):
        ckv.ckv_paged_attention_q4(c.cfg, cache, table, lens, cu, c.q, out, ws)
        assert ckv.ckv_read_device_status(ws)[0] == 2
    ckv.ckv_set_wait_limit_us(0)
    ws.zero_()
    ckv.ckv_paged_attention_q4(c.cfg, cache, table, lens, cu, c.q, out, ws)
    assert ckv.ckv_read_device_status(ws) == (0, 0)
    for s, (L, n) in enumerate(zip(c.lens, c.new)):
        a = int(c.cu[s])
        o, _, tol, _ = ref.rows(c.q[a:a + n], c.k[s], c.v[s], torch.arange(L - n, L))
        ref.assert_close(out[a:a + n], o, tol, f"sequence {s}")


@pytest.mark.parametrize("new", [1, 2, 4, 8])
def test_few_rows_wait_for_nothing(one_microsecond, new):  # noqa: F811
    Paged4(config(), (3000, 700, 90), (new,) * 3, 32, seed=21).check()


@pytest.mark.parametrize("lens,new", [((90,), 40), ((300,) * 60, 20), ((200,) * 60, 5), ((130, 60), 40), ((1000,) * 7, 300)])
def test_copies_of_pages_land_before_a_block_leaves(one_microsecond, lens, new):  # noqa: F811
    c = Paged4(config(), lens, (new,) * len(lens), 16, seed=22)
    cache, wss = ckv.PagedCacheQ4(c.pages, 16), [ckv.new_attention_workspace(c.cfg) for _ in range(2)]
    table, n, cu = arguments(c)
    out, o_good = torch.zeros_like(c.q), torch.zeros_like(c.q)
    ckv.ckv_set_wait_limit_us(0)
    ckv.ckv_paged_attention_q4(c.cfg, cache, table, n, cu, c.q, o_good, wss[1])
    want = o_good.clone()

    def bad():
        wss[0].zero_()
        ckv.ckv_paged_attention_q4(c.cfg, cache, table, n, cu, c.q, out, wss[0])
        return wss[0]

    def good():
        o_good.zero_()
        ckv.ckv_paged_attention_q4(c.cfg, cache, table, n, cu, c.q, o_good, wss[1])
        return wss[1]

    def check_good():
        assert torch.equal(o_good, want)

    calls_after_calls_that_gave_up(bad, good, lambda: torch.equal(out, want), check_good)
