"""Lengths and tables at the ends of their ranges in the serving operators."""
import numpy as np
import pytest
import torch

from oracle import serve_ops as S
from test_gpu_cache import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,page,shift", [(1, 8, 0), (2, 16, 1), (3, 24, 4)])
@pytest.mark.parametrize("over", [1, 3, 4, 10 ** 6, 2 ** 31 - 1])
def test_append_keeps_the_slots_of_tokens_that_have_one(over, H, page, shift):
    """A length beyond the table: the tokens that still have a slot go there, no other slot changes."""
    from paper_2410_17765_b200 import binding

    Q = 4
    c = Case([4 * page, 20], H, 8, page, Q=Q, seed=page)
    most = c.table.shape[1] * page
    behind = c.table_np < 0                  # the table's last pages, which the sequences do not have yet
    c.table_np[behind] = [p for p in range(c.k.shape[0]) if p not in c.table_np][:int(behind.sum())]
    c.table = torch.from_numpy(c.table_np).cuda()
    long = min(most + over, 2 ** 31 - 1)
    lens = torch.tensor([long, 20], dtype=torch.int32, device="cuda")
    wide = torch.randn(2, Q, H * 8 + 8, device="cuda").to(torch.bfloat16)
    k = wide[:, :, shift:shift + H * 8].unflatten(2, (H, 8))
    want, want_a = c.k.clone(), c.acc.clone()
    for b, n in enumerate((long, 20)):
        for j in range(Q):
            slot = n - Q + j
            if slot < most:
                page_of, at = S.places(c.table_np[b], page, slot + 1)
                want[int(page_of[-1]), int(at[-1])] = k[b, j]
                want_a[int(page_of[-1]), :, int(at[-1])] = 0
    binding.cache_append(c.cache(), k, k, c.table, lens, dev_status=c.status)
    assert int(c.status.item()) == 1
    assert torch.equal(torch.nan_to_num(c.k, 99.0), torch.nan_to_num(want, 99.0)) and torch.equal(torch.nan_to_num(c.acc, 99.0), torch.nan_to_num(want_a, 99.0))
