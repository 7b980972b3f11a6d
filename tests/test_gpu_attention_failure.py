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
