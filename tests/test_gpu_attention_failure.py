"""Bounded waits of the attention kernels: a limit that runs out is reported, every role leaves, and the
context serves the next call (with the workspace zeroed again, as the header asks)."""
import pytest
import torch

import paper_2508_02401_gb300 as ckv
from tests import attention_ref as ref
from tests.test_gpu_paged_attention import Paged
from tests.test_gpu_prefill_attention import check, config, normal

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    if not torch.cuda.is_available():
        pytest.skip("needs a GPU")
    ckv.load()


@pytest.fixture
def one_microsecond():
    ckv.ckv_set_wait_limit_us(1)  # the first loads outlast it
    yield
    ckv.ckv_set_wait_limit_us(0)


@pytest.mark.parametrize("lens", [(900,), (4000, 300, 17)])
def test_prompts(one_microsecond, lens):
    cfg, T = config(), sum(lens)
    q, k, v = normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2), normal(T, 2, 128, seed=3)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    ws, out = ckv.new_attention_workspace(cfg), torch.zeros_like(q)
    for _ in range(3):
        ckv.ckv_prefill_attention(cfg, ckv.Batch(cu), q, k, v, out, ws)
        assert ckv.ckv_read_device_status(ws)[0] == 2
    ckv.ckv_set_wait_limit_us(0)
    check(cfg, lens, q, k, v)


@pytest.mark.parametrize("new", [1, 2, 4, 8, 70])  # 4, 8 and 16 rows a unit, and the kernel for 256
def test_new_tokens(one_microsecond, new):
    c = Paged(config(), (3000, 700, 90), (new,) * 3, 32, seed=21)
    ws = ckv.new_attention_workspace(c.cfg)
    cache = ckv.PagedCache(c.k_pages, c.v_pages)
    table, lens, cu = (torch.as_tensor(x, dtype=torch.int32, device="cuda") for x in (c.table, c.lens, c.cu))
    out = torch.zeros_like(c.q)
    for _ in range(3):
        ckv.ckv_paged_attention(c.cfg, cache, table, lens, cu, c.q, out, ws)
        assert ckv.ckv_read_device_status(ws)[0] == 2
    ckv.ckv_set_wait_limit_us(0)
    ws.zero_()
    ckv.ckv_paged_attention(c.cfg, cache, table, lens, cu, c.q, out, ws)
    assert ckv.ckv_read_device_status(ws) == (0, 0)
    for s, (L, n) in enumerate(zip(c.lens, c.new)):
        a = int(c.cu[s])
        o, _, tol, _ = ref.rows(c.q[a:a + n], c.k[s], c.v[s], torch.arange(L - n, L))
        ref.assert_close(out[a:a + n], o, tol, f"sequence {s}")


def calls_after_calls_that_gave_up(bad, good, right, check_good):
    """A call that gave up and, at once behind it, one that may take over its CTAs' shared memory: no load of the first
    may still be on its way there.  Loaders whose tiles fit their ring never wait themselves."""
    for _ in range(20):
        ckv.ckv_set_wait_limit_us(1)
        ws = bad()
        ckv.ckv_set_wait_limit_us(0)
        ws_good = good()
        # (each wait of a call that finds its few tiles in L2 may be over within the limit: then its result is right)
        code = ckv.ckv_read_device_status(ws)[0]
        assert code == 2 or (code == 0 and right())
        assert ckv.ckv_read_device_status(ws_good) == (0, 0)
        check_good()


@pytest.mark.parametrize("lens", [(1,), (100,), (129, 300), (256,) * 40, (700,) * 20])
def test_copies_of_prompts_land_before_a_block_leaves(one_microsecond, lens):
    cfg, T = config(), sum(lens)
    q, k, v = normal(T, 8, 128, seed=1), normal(T, 2, 128, seed=2), normal(T, 2, 128, seed=3)
    cu = [0]
    for n in lens:
        cu.append(cu[-1] + n)
    batch, wss = ckv.Batch(cu), [ckv.new_attention_workspace(cfg) for _ in range(2)]
    out, o_good = torch.zeros_like(q), torch.zeros_like(q)
    ckv.ckv_set_wait_limit_us(0)
    ckv.ckv_prefill_attention(cfg, batch, q, k, v, o_good, wss[1])
    want = o_good.clone()

    def bad():
        wss[0].zero_()
        ckv.ckv_prefill_attention(cfg, batch, q, k, v, out, wss[0])
        return wss[0]

    def good():
        o_good.zero_()
        ckv.ckv_prefill_attention(cfg, batch, q, k, v, o_good, wss[1])
        return wss[1]

    def check_good():
        assert torch.equal(o_good, want)

    calls_after_calls_that_gave_up(bad, good, lambda: torch.equal(out, want), check_good)


@pytest.mark.parametrize("lens,new", [((90,), 1), ((300,) * 200, 1), ((200,) * 60, 2), ((130,) * 60, 4), ((130, 60), 40)])
def test_copies_of_pages_land_before_a_block_leaves(one_microsecond, lens, new):
    c = Paged(config(), lens, (new,) * len(lens), 16, seed=22)
    cache, wss = ckv.PagedCache(c.k_pages, c.v_pages), [ckv.new_attention_workspace(c.cfg) for _ in range(2)]
    table, n, cu = (torch.as_tensor(x, dtype=torch.int32, device="cuda") for x in (c.table, c.lens, c.cu))
    out, o_good = torch.zeros_like(c.q), torch.zeros_like(c.q)
    ckv.ckv_set_wait_limit_us(0)
    ckv.ckv_paged_attention(c.cfg, cache, table, n, cu, c.q, o_good, wss[1])
    want = o_good.clone()

    def bad():
        wss[0].zero_()
        ckv.ckv_paged_attention(c.cfg, cache, table, n, cu, c.q, out, wss[0])
        return wss[0]

    def good():
        o_good.zero_()
        ckv.ckv_paged_attention(c.cfg, cache, table, n, cu, c.q, o_good, wss[1])
        return wss[1]

    def check_good():
        assert torch.equal(o_good, want)

    calls_after_calls_that_gave_up(bad, good, lambda: torch.equal(out, want), check_good)
