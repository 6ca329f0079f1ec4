"""Layouts that the serving entry points refuse on the host, since two threads would write to one place."""
import pytest
import torch

from paper_2410_17765_b200 import binding
from test_host_serve_ops import P, attend, cache, calls, evict, lib, seqs, tokens  # noqa: F401

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


@pytest.mark.parametrize("layout,code", [(dict(seq=0), -2), (dict(seq=256), -2), (dict(token=128), -2), (dict(token=64, head=64), -2), (dict(seq=511), -2), (dict(seq=64, token=192, head=320), -2),
                                         (dict(seq=1 << 60), -7)], ids=str)
def test_outputs_must_not_overlap(lib, layout, code):
    """Three sequences of two tokens of four heads of 64; queries may overlap (a batch of one row expanded)."""
    c, s = cache(), seqs()
    need = lib.cpmtp_cache_attend_workspace_bytes(c, s, 4)
    assert lib.cpmtp_cache_attend(c, s, attend(out=tokens(**layout)), P, need, None, None) == code
    if NO_GPU:
        assert lib.cpmtp_cache_attend(c, s, attend(q=tokens(seq=0)), P, need, None, None) in (-5, -6)


@pytest.mark.skipif(not NO_GPU, reason="the addresses are made up")
@pytest.mark.parametrize("layout", [dict(), dict(seq=1024), dict(seq=2048, token=64, head=128), dict(seq=64, token=192, head=384)], ids=str)
def test_outputs_that_lie_apart_are_taken(lib, layout):
    c, s = cache(), seqs()
    need = lib.cpmtp_cache_attend_workspace_bytes(c, s, 4)
    assert lib.cpmtp_cache_attend(c, s, attend(out=tokens(**layout)), P, need, None, None) in (-5, -6)


@pytest.mark.parametrize("off", [-8, -4, 0, 4, 8])
def test_new_lengths_must_not_overlap_the_old_ones(lib, off):
    c, s = cache(), seqs()
    need = lib.cpmtp_cache_evict_workspace_bytes(c, s, 32)
    assert lib.cpmtp_cache_evict(c, s, evict(lens_out=P + off), P, need, None, None) == -2
    if NO_GPU:
        for apart in (-12, 12):
            assert lib.cpmtp_cache_evict(c, s, evict(lens_out=P + apart), P, need, None, None) in (-5, -6)
