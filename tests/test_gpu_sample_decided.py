"""The comparisons with the fp64 restatement pass over rows whose decisions lie next to a border; here it is counted how many they are."""
import numpy as np
import pytest
import torch

import test_gpu_sample as T
from oracle import serve_ops as S

pytestmark = pytest.mark.gpu


@pytest.fixture
def share(monkeypatch):
    """The share of rows that were compared."""
    gaps, sample = [], S.sample

    def counted(*args):
        r = sample(*args)
        gaps.append(r["gap"])
        return r

    monkeypatch.setattr(S, "sample", counted)
    return lambda: float(np.mean([g > 2.0 ** -31 for g in gaps]))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("how", T.FILTERS, ids=str)
def test_nearly_all_rows_of_random_logits_are_compared(how, dtype, share):
    for N, V in ((40, 1000), (20, 4097), (12, 32003), (3, 128256)):
        x, u = T.draw(N, V, V + 1, dtype)
        T.check(x, u, given=x.argmax(1).int(), sure=False, **how)
    assert share() >= 0.9


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nearly_all_rows_with_settings_of_their_own_are_compared(dtype, share):
    N = 100
    x, u = T.draw(N, 5003, 21, dtype)
    r = torch.rand(4, N, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    T.check(x, u, T=torch.where(r[0] < 0.2, 0.0, r[0] * 2), k=((r[1] - 0.3) * 100).to(torch.int32), p=r[2] * 1.5, min_p=r[3] * 0.2 - 0.05, sure=False)
    assert share() >= 0.9


@pytest.mark.parametrize("N,how", [(700, dict(k=30, p=0.9)), (150, dict(p=0.8)), (40, dict(k=1500, min_p=1e-4)), (8, dict(p=0.999)), (300, dict(p=2.0 ** -7))], ids=str)
def test_nearly_all_rows_of_many_sizes_of_batches_are_compared(N, how, share):
    x, u = T.draw(N, 2049, N + 1, torch.bfloat16)
    T.check(x, u, sure=False, **how)
    assert share() >= 0.9
