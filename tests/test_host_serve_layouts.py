"""Layouts that the serving entry points refuse on the host, since two threads would write to one place."""
import pytest
import torch

from paper_2410_17765_b200 import binding
from test_host_serve_ops import attend, cache, calls, evict, lib, seqs, tokens  # noqa: F401

NO_GPU = not torch.cuda.is_available()


# ten pages of two heads of sixteen slots
OVERLAPPING_ACC = [dict(acc_page=16, acc_head=16), dict(acc_page=24, acc_head=16), dict(acc_page=16, acc_head=24), dict(acc_page=16, acc_head=152), dict(acc_page=31, acc_head=16)]
APART_ACC = [dict(acc_page=32, acc_head=16), dict(acc_page=16, acc_head=160), dict(acc_page=33, acc_head=17), dict(pages=1, acc_page=16, acc_head=16),
             dict(H=1, acc_page=16, acc_head=16), dict(pages=1, H=1, acc_page=16, acc_head=16)]


@pytest.mark.parametrize("layout", OVERLAPPING_ACC, ids=str)
def test_pages_and_heads_of_acc_must_not_overlap(lib, layout):
    assert set(calls(lib, cache(**layout), seqs())) == {-2}
    assert lib.cpmtp_cache_attend_workspace_bytes(cache(**layout), seqs(), 4) == 0
    # without acc its distances mean nothing
    assert lib.cpmtp_cache_attend_workspace_bytes(cache(acc=None, **layout), seqs(), 4) > 0


@pytest.mark.parametrize("layout", APART_ACC, ids=str)
def test_pages_and_heads_of_acc_that_lie_apart_are_taken(lib, layout):
    assert lib.cpmtp_cache_attend_workspace_bytes(cache(**layout), seqs(), 4) > 0


FAR = 1 << 37


@pytest.mark.parametrize("layout", [dict(pages=2 ** 31 - 1, k_page=FAR, k_head=FAR + 64), dict(pages=2 ** 31 - 1, v_page=FAR), dict(pages=2 ** 31 - 1, acc_page=FAR, acc_head=FAR + 16),
                                    dict(pages=2 ** 31 - 1, H=65535, k_page=FAR, k_head=FAR + 128)], ids=str)
def test_spans_beyond_64_bits_are_refused(lib, layout):
    """Offsets of the last pages would not fit, and what the pages span is not known to overlap or not."""
    assert set(calls(lib, cache(**layout), seqs())) == {-7}
    assert lib.cpmtp_cache_attend_workspace_bytes(cache(**layout), seqs(), 4) == 0
