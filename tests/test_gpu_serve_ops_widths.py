"""Tables much wider than the sequences, as a server has them that captures its steps: results are those of a table that just fits, bit for bit."""
import numpy as np
import pytest
import torch

from test_gpu_cache import Case

pytestmark = pytest.mark.gpu


def widened(c, width, fill=-7):
    return torch.nn.functional.pad(c.table, (0, width - c.table.shape[1]), value=fill)


@pytest.mark.parametrize("slots", [4096, 131072, 1 << 20])
@pytest.mark.parametrize("lens,Q,Hq,page", [([300, 1, 0, 129], 1, 4, 16), ([700, 131, 20], 5, 8, 64), ([3000], 9, 8, 24), ([1000] * 20, 2, 2, 128)])
def test_attend(lens, Q, Hq, page, slots):
    from paper_2410_17765_b200 import binding

    c = Case(lens, 2, 64, page, Q=Q, Hq=Hq, seed=Q)
    start = c.acc.clone()
    want = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, want_lse=True, dev_status=c.status)
    want_acc = c.acc.clone()
    c.acc.copy_(start)
    got = binding.cache_attend(c.cache(), c.q, widened(c, slots // page), c.lens_t, want_lse=True, dev_status=c.status)
    assert int(c.status.item()) == 0
    assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
    assert torch.equal(torch.nan_to_num(c.acc, 9.0), torch.nan_to_num(want_acc, 9.0))


@pytest.mark.parametrize("slots", [8192, 131072, 600000, 1 << 20])           # (keys of a head in one block's, in eight blocks', in no shared memory)
@pytest.mark.parametrize("lens,budget,recent", [([5000, 300, 0, 1001], 1000, 100), ([2048] * 30, 512, 0)])
def test_evict(lens, budget, recent, slots):
    from paper_2410_17765_b200 import binding

    page = 16
    c = Case(lens, 2, 16, page, more=-(-budget // page), seed=budget)
    start = [t.clone() for t in (c.k, c.v, c.acc)]
    want = binding.cache_evict(c.cache(), c.table, c.lens_t, c.table_out, budget, recent=recent, dev_status=c.status)
    after = [t.clone() for t in (c.k, c.v, c.acc)]
    for t, s in zip((c.k, c.v, c.acc), start):
        t.copy_(s)
    got = binding.cache_evict(c.cache(), widened(c, slots // page), c.lens_t, widened_out(c, slots // page), budget, recent=recent, dev_status=c.status)
    assert int(c.status.item()) == 0
    assert torch.equal(got["lens"], want["lens"]) and torch.equal(got["kept"], want["kept"])
    assert all(torch.equal(torch.nan_to_num(t, 9.0), torch.nan_to_num(a, 9.0)) for t, a in zip((c.k, c.v, c.acc), after))


def widened_out(c, width):
    return torch.nn.functional.pad(c.table_out, (0, width - c.table_out.shape[1]), value=-7)


def test_append():
    from paper_2410_17765_b200 import binding

    c = Case([300, 20, 4], 2, 64, 16, Q=4, fresh=[4, 1, 4])
    k = torch.from_numpy(np.random.default_rng(1).normal(size=(3, 4, 2, 64)).astype(np.float32)).to(torch.bfloat16).cuda()
    start = c.k.clone()
    binding.cache_append(c.cache(), k, k, c.table, c.lens_t, q_lens=c.fresh_t, dev_status=c.status)
    want = c.k.clone()
    c.k.copy_(start)
    binding.cache_append(c.cache(), k, k, widened(c, 1 << 16), c.lens_t, q_lens=c.fresh_t, dev_status=c.status)
    assert int(c.status.item()) == 0 and torch.equal(torch.nan_to_num(c.k, 9.0), torch.nan_to_num(want, 9.0))
