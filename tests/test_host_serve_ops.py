"""CPU-only checks of the serving entry points: structure layouts, workspaces, and that bad arguments are rejected before a GPU is
touched."""
import ctypes
import os
import re

import pytest
import torch

from paper_2410_17765_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P, ODD = 4096, 4097
NO_GPU = not torch.cuda.is_available()


@pytest.fixture(scope="module")
def lib():
    build.build()
    return binding.load_library()


def test_structures_have_the_headers_fields_in_order():
    header = open(os.path.join(ROOT, "include", "cpmtp.h")).read()

    def names(struct):
        body = re.sub(r"/\*.*?\*/", "", re.search(r"typedef struct %s \{(.*?)\} %s;" % (struct, struct), header, re.S).group(1), flags=re.S)
        out = []
        for decl in body.split(";"):
            words = decl.replace("*", " ").replace(",", " ").split()
            out += words[2:] if words[:1] == ["const"] else words[1:]
        return out

    for struct, cls in (("cpmtp_cache", binding.CCache), ("cpmtp_cache_seqs", binding.CCacheSeqs), ("cpmtp_tokens", binding.CTokens),
                        ("cpmtp_attend_args", binding.CAttendArgs), ("cpmtp_evict_args", binding.CEvictArgs), ("cpmtp_sample_args", binding.CSampleArgs)):
        assert names(struct) == [f[0] for f in cls._fields_], struct
    assert re.search(r"#define CPMTP_CACHE_MAX_D (\d+)", header).group(1) == str(binding.CACHE_MAX_D)


def cache(**kw):
    a = dict(k=P, v=P, acc=P, pages=10, page_slots=16, H=2, D=64, k_page=2048, k_slot=128, k_head=64, v_page=2048, v_slot=128, v_head=64, acc_page=32, acc_head=16)
    a.update(kw)
    return binding.CCache(*[a[f[0]] for f in binding.CCache._fields_])


def seqs(**kw):
    a = dict(table=P, lens=P, q_lens=None, ld_table=4, B=3, width=4, Q=2, unused=0)
    a.update(kw)
    return binding.CCacheSeqs(*[a[f[0]] for f in binding.CCacheSeqs._fields_])


def tokens(**kw):
    a = dict(data=P, seq=512, token=256, head=64)
    a.update(kw)
    return binding.CTokens(*[a[f[0]] for f in binding.CTokens._fields_])


def attend(**kw):
    a = dict(q=tokens(), out=tokens(), lse=None, Hq=4, scale=0.125)
    a.update(kw)
    return binding.CAttendArgs(*[a[f[0]] for f in binding.CAttendArgs._fields_])


def evict(**kw):
    a = dict(table_out=P, ld_table_out=2, budget=32, recent=4, lens_out=2 * P, kept=None)
    a.update(kw)
    return binding.CEvictArgs(*[a[f[0]] for f in binding.CEvictArgs._fields_])


def sample(**kw):
    a = dict.fromkeys([f[0] for f in binding.CSampleArgs._fields_], None)
    a.update(logits=P, ld=100, N=4, V=100, type=binding.F32, top_k=0, temperature=1.0, top_p=1.0, min_p=0.0, unused=0, uniform=P, tokens=P)
    a.update(kw)
    return binding.CSampleArgs(*[a[f[0]] for f in binding.CSampleArgs._fields_])


BAD_CACHES = [(dict(pages=0), -2), (dict(page_slots=12), -2), (dict(page_slots=0), -2), (dict(page_slots=65544), -2), (dict(H=0), -2), (dict(D=0), -2), (dict(D=60), -2),
              (dict(D=136), -7), (dict(k_slot=56), -2), (dict(v_head=32), -2), (dict(k_page=1024), -2), (dict(k_head=68, k_slot=136), -3), (dict(v_page=1 << 40), -7),
              (dict(k_slot=-128), -2), (dict(acc_head=8), -2), (dict(acc_page=8), -2)]
BAD_SEQS = [(dict(B=-1), -2), (dict(width=-1), -2), (dict(ld_table=3), -2), (dict(Q=-1), -2), (dict(B=70000), -7), (dict(width=1 << 27, ld_table=1 << 27), -7)]
BAD_DATA = [(dict(k=None), {}, -1), (dict(v=None), {}, -1), (dict(k=P + 8), {}, -3), (dict(acc=P + 2), {}, -3), ({}, dict(table=None), -1), ({}, dict(lens=None), -1),
            ({}, dict(lens=ODD), -3), ({}, dict(table=P + 2), -3), ({}, dict(q_lens=P + 1), -3)]


def calls(lib, c, s):
    """The three calls on a cache, with arguments that are right otherwise."""
    yield lib.cpmtp_cache_append(c, s, tokens(), tokens(), None, None)
    yield lib.cpmtp_cache_attend(c, s, attend(), P, 1 << 40, None, None)
    yield lib.cpmtp_cache_evict(c, s, evict(), P, 1 << 40, None, None)


@pytest.mark.parametrize("bad,code", BAD_CACHES, ids=str)
def test_caches_are_checked(lib, bad, code):
    assert set(calls(lib, cache(**bad), seqs())) == {code}
    assert lib.cpmtp_cache_attend_workspace_bytes(cache(**bad), seqs(), 4) == 0
    assert lib.cpmtp_cache_evict_workspace_bytes(cache(**bad), seqs(), 32) == 0


@pytest.mark.parametrize("bad,code", BAD_SEQS, ids=str)
def test_sequences_are_checked(lib, bad, code):
    assert set(calls(lib, cache(), seqs(**bad))) == {code}
    assert lib.cpmtp_cache_attend_workspace_bytes(cache(), seqs(**bad), 4) == 0


@pytest.mark.parametrize("c,s,code", BAD_DATA, ids=str)
def test_addresses_are_checked(lib, c, s, code):
    assert set(calls(lib, cache(**c), seqs(**s))) == {code}


def test_structures_may_not_be_missing(lib):
    c, s = cache(), seqs()
    assert lib.cpmtp_cache_append(None, s, tokens(), tokens(), None, None) == -1
    assert lib.cpmtp_cache_append(c, None, tokens(), tokens(), None, None) == -1
    assert lib.cpmtp_cache_append(c, s, None, tokens(), None, None) == -1
    assert lib.cpmtp_cache_attend(c, s, None, P, 1 << 40, None, None) == -1
    assert lib.cpmtp_cache_evict(c, s, None, P, 1 << 40, None, None) == -1
    assert lib.cpmtp_sample_logits(None, None, None) == -1


def test_append_arguments_are_checked(lib):
    c, s = cache(), seqs()
    for bad, code in ((dict(data=None), -1), (dict(data=ODD), -3), (dict(token=32), -2), (dict(head=32), -2), (dict(seq=-1), -2)):
        assert lib.cpmtp_cache_append(c, s, tokens(**bad), tokens(), None, None) == code
        assert lib.cpmtp_cache_append(c, s, tokens(), tokens(**bad), None, None) == code
    assert lib.cpmtp_cache_append(c, s, tokens(), tokens(), ODD, None) == -3
    assert lib.cpmtp_cache_append(c, seqs(B=0), None, None, None, None) == 0
    assert lib.cpmtp_cache_append(c, seqs(Q=0), None, None, None, None) == 0


def test_attend_arguments_are_checked(lib):
    c, s = cache(), seqs()
    need = lib.cpmtp_cache_attend_workspace_bytes(c, s, 4)
    # with acc the scores of every row and slot are kept: 6 units of a tile of 16 rows
    assert need >= 6 * 16 * 128 * 4 > lib.cpmtp_cache_attend_workspace_bytes(cache(acc=None), s, 4) - 148 * 2 * 16 * 520
    for bad, code in ((dict(Hq=3), -2), (dict(Hq=0), -2), (dict(scale=float("inf")), -2), (dict(scale=float("nan")), -2), (dict(q=tokens(data=None)), -1),
                      (dict(out=tokens(data=None)), -1), (dict(q=tokens(data=ODD)), -3), (dict(out=tokens(head=8)), -2), (dict(lse=P + 2), -3)):
        assert lib.cpmtp_cache_attend(c, s, attend(**bad), P, need, None, None) == code, bad
    assert lib.cpmtp_cache_attend(c, s, attend(), None, need, None, None) == -1
    assert lib.cpmtp_cache_attend(c, s, attend(), P + 16, need, None, None) == -3
    assert lib.cpmtp_cache_attend(c, s, attend(), P, need - 1, None, None) == -4
    assert lib.cpmtp_cache_attend(c, s, attend(), P, need, ODD, None) == -3
    assert lib.cpmtp_cache_attend(c, seqs(B=0), attend(), None, 0, None, None) == 0
    # more tiles than a 31-bit count holds
    many = seqs(B=60000, width=1 << 20, ld_table=1 << 20, Q=64)
    assert lib.cpmtp_cache_attend_workspace_bytes(c, many, 4) == 0
    assert lib.cpmtp_cache_attend(c, many, attend(), P, 1 << 60, None, None) == -7


def test_evict_arguments_are_checked(lib):
    c, s = cache(), seqs()
    need = lib.cpmtp_cache_evict_workspace_bytes(c, s, 32)
    assert need >= 3 * 2 * 32 * 4
    for bad, code in ((dict(budget=0), -2), (dict(recent=-1), -2), (dict(recent=33), -2), (dict(ld_table_out=1), -2), (dict(table_out=None), -1), (dict(lens_out=None), -1),
                      (dict(lens_out=P), -2), (dict(kept=ODD), -3), (dict(table_out=P + 2), -3), (dict(lens_out=P + 2), -3)):
        assert lib.cpmtp_cache_evict(c, s, evict(**bad), P, need, None, None) == code, bad
    assert lib.cpmtp_cache_evict(cache(acc=None), s, evict(), P, need, None, None) == -1
    assert lib.cpmtp_cache_evict(c, s, evict(), P, need - 1, None, None) == -4
    assert lib.cpmtp_cache_evict(c, s, evict(), None, need, None, None) == -1
    if NO_GPU:                                   # with `kept` none is needed
        assert lib.cpmtp_cache_evict(c, s, evict(kept=P), None, 0, None, None) in (-5, -6)
    assert lib.cpmtp_cache_evict(c, seqs(B=0), evict(), None, 0, None, None) == 0


def test_sample_arguments_are_checked(lib):
    nan, inf = float("nan"), float("inf")
    for bad, code in ((dict(N=-1), -2), (dict(V=0), -2), (dict(ld=99), -2), (dict(type=2), -2), (dict(V=(1 << 24) + 1, ld=1 << 25), -7), (dict(temperature=-1.0), -2),
                      (dict(temperature=nan), -2), (dict(temperature=inf), -2), (dict(top_p=-0.5), -2), (dict(top_p=nan), -2), (dict(min_p=nan), -2), (dict(top_k=-1), -2),
                      (dict(logits=None), -1), (dict(uniform=None), -1), (dict(tokens=None), -1), (dict(given=P), -1), (dict(logits=P + 2), -3), (dict(uniform=ODD), -3),
                      (dict(kept=P + 2), -3), (dict(temperatures=P + 1), -3)):
        assert lib.cpmtp_sample_logits(sample(**bad), None, None) == code, bad
    assert lib.cpmtp_sample_logits(sample(), ODD, None) == -3
    assert lib.cpmtp_sample_logits(sample(N=0, logits=None, uniform=None, tokens=None), None, None) == 0


@pytest.mark.skipif(not NO_GPU, reason="the addresses are made up")
def test_right_arguments_reach_the_device(lib):
    c, s = cache(), seqs()
    assert all(rc in (-5, -6) for rc in calls(lib, c, s))
    assert lib.cpmtp_sample_logits(sample(), None, None) in (-5, -6)


def test_caches_of_the_binding_are_checked():
    k = torch.zeros(6, 16, 2, 64, dtype=torch.bfloat16)
    acc = torch.zeros(6, 2, 16)
    c = binding.PagedCache(k, k.clone(), acc)
    assert c.page_slots == 16 and c.heads == 2
    hnd = torch.zeros(6, 2, 16, 64, dtype=torch.bfloat16).transpose(1, 2)
    assert binding.PagedCache(hnd, hnd)._plain.k_head == 16 * 64
    one = binding.PagedCache(k[:1, :, :1], k[:1, :, :1])._plain           # distances of dimensions of size one do not matter
    assert (one.k_page, one.k_head) == (64, 64)
    for bad in ((k.float(), k), (k, k[:, :8]), (k[0], k[0]), (k[:, :12], k[:, :12]), (k[..., :60], k[..., :60]), (k[:0], k[:0]), (k.transpose(2, 3), k.transpose(2, 3)),
                (k, k, acc.double()), (k, k, acc[:, :1]), (k, k, acc.transpose(1, 2)), (torch.zeros(2, 16, 2, 136, dtype=torch.bfloat16),) * 2,
                (torch.zeros(1 + 2 * 16 * 2 * 64, dtype=torch.bfloat16)[1:].view(2, 16, 2, 64),) * 2, (torch.zeros(2, 16, 2, 68, dtype=torch.bfloat16)[..., :64],) * 2):
        with pytest.raises(binding.CpmtpError):
            binding.PagedCache(*bad)
