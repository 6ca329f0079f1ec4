"""Loads that never come (left out by the test hook) in the middle of a share: attention over the cache gives up with products, tiles and parts under way."""
import pytest
import torch

from test_gpu_cache import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("skip", [3, 4, 5, 6, 9, 14])
def test_waits_between_tiles_give_up_and_the_library_stays_usable(skip, accumulate):
    """Nine tiles or more to every share, of one unit or two: load 2 i + 1 is that of tile i of keys, 2 i + 2 that of its values."""
    from paper_2410_17765_b200 import binding

    c = Case([60000, 30000], 2, 64, 64, Hq=4, seed=5)
    tiles = 2 * sum(-(-n // 128) for n in c.lens)
    assert tiles // torch.cuda.get_device_properties(0).multi_processor_count >= 9
    start = c.acc.clone()

    def call():
        return binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=accumulate, dev_status=c.status)["out"]

    want, want_acc = call(), c.acc.clone()
    c.acc.copy_(start)
    torch.cuda.synchronize()
    with binding.knobs(CPMTP_WAIT_LIMIT_US=20000, CPMTP_TEST_SKIP_LOAD=skip):
        call()
        torch.cuda.synchronize()
    assert int(c.status.item()) == 2
    c.status.zero_()
    c.acc.copy_(start)
    got = call()
    assert int(c.status.item()) == 0 and torch.equal(got, want)
    assert torch.equal(torch.nan_to_num(c.acc, 9.0), torch.nan_to_num(want_acc, 9.0))
