"""CPU-only checks of what the binding's optimiser hands to the library: a stand-in for the library records the descriptors."""
import ctypes
import gc
import time

import pytest
import torch

from paper_2410_17765_b200 import binding


class Recorder:
    """In the library's place: the descriptors of the last call, as a list of dicts."""

    def __init__(self):
        self.calls = []

    def cpmtp_adamw_step(self, address, count, hyper, stream):
        table = (binding.CAdamWTensor * count).from_address(address)
        self.calls.append([{f[0]: getattr(t, f[0]) for f in t._fields_} for t in table])
        return 0

    @property
    def last(self):
        return self.calls[-1]


@pytest.fixture
def lib(monkeypatch):
    rec = Recorder()
    monkeypatch.setattr(binding, "load_library", lambda: rec)
    monkeypatch.setattr(binding, "_device", lambda t: t.get_device())       # (-1: the CPU, here as good as any)
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    return rec


def check(lib, opt, grads):
    """The last call named exactly the tensors that the optimiser's lists hold now."""
    columns = dict(param=opt.params, grad=grads, master=opt.master, m=opt.m, v=opt.v)
    if opt.bits == 8:
        columns.update(m_exp=opt.m_exp, v_exp=opt.v_exp)
    for i, got in enumerate(lib.last):
        for name, tensors in columns.items():
            assert (got[name] or 0) == (0 if tensors[i] is None else tensors[i].data_ptr()), (i, name)
        assert got["numel"] == opt.params[i].numel()
        assert got["param_type"] == binding._TYPES[opt.params[i].dtype]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
def test_a_step_names_the_tensors_that_are_there_now(lib, bits, master):
    sizes = [300, 7, 512]
    params = [torch.zeros(n, dtype=torch.bfloat16) for n in sizes]
    grads = [torch.zeros(n, dtype=torch.bfloat16) for n in sizes]
    opt = binding.AdamW(params, bits=bits, master=master)
    opt.step(grads, 1, lr=0.1)
    check(lib, opt, grads)
    params[1].data = torch.ones(7, dtype=torch.bfloat16)                    # what a module's .to() does
    opt.step(grads, 2, lr=0.1)
    check(lib, opt, grads)
    for name in ["m", "v"] + (["m_exp", "v_exp"] if bits == 8 else []) + (["master"] if master else []):
        setattr(opt, name, [t.clone() for t in getattr(opt, name)])         # a restored state
        opt.step(grads, 3, lr=0.1)
        check(lib, opt, grads)
        with pytest.raises(TypeError):                                      # not one by one, which would go unnoticed
            getattr(opt, name)[2] = getattr(opt, name)[2].clone()
        getattr(opt, name)[0].data = torch.zeros(0)                         # the memory that a step writes stays what it was
        opt.step(grads, 4, lr=0.1)
        check(lib, opt, grads)
        assert getattr(opt, name)[0].numel() > 0
    if master:
        opt.master = [None, *opt.master[1:]]
        opt.step(grads, 5, lr=0.1)
        check(lib, opt, grads)
    opt.params[0] = torch.zeros(300, dtype=torch.bfloat16)
    opt.step(grads, 6, lr=0.1)
    check(lib, opt, grads)


def test_memory_that_the_descriptors_name_is_held_until_they_are_renewed(lib):
    """Else another tensor could come to lie there, with the same address and another size."""
    p = torch.zeros(1 << 16)
    opt = binding.AdamW([p])
    was = [p.data_ptr(), opt.m[0].data_ptr()]
    p.data = torch.zeros(0)
    gc.collect()
    fresh = [torch.zeros(1 << 16) for _ in range(16)]
    assert all(t.data_ptr() not in was for t in fresh)


def test_states_that_were_given_are_held_as_they_were(lib):
    p, m = torch.zeros(300), torch.zeros(300)
    opt = binding.AdamW([p], state=dict(m=[m], v=[torch.zeros(300)]))
    was = m.data_ptr()
    m.data = torch.zeros(300)
    opt.step([torch.zeros(300)], 1, lr=0.1)
    assert lib.last[0]["m"] == was == opt.m[0].data_ptr()


def test_a_changed_type_is_taken_up(lib):
    p = torch.zeros(300)
    opt = binding.AdamW([p])
    opt.step([torch.zeros(300)], 1, lr=0.1)
    assert lib.last[0]["param_type"] == binding.F32
    p.data = p.to(torch.bfloat16)
    opt.step([torch.zeros(300)], 2, lr=0.1)
    assert lib.last[0]["param_type"] == binding.BF16 and lib.last[0]["grad_type"] == binding.F32


def test_tensors_that_no_longer_fit_are_refused(lib):
    def fresh(bits=32):
        p = [torch.zeros(64), torch.zeros(64)]
        opt = binding.AdamW(p, bits=bits)
        opt.step([torch.zeros(64)] * 2, 1, lr=0.1)
        return p, opt

    def replaced_by_a_shorter_one(p, opt):
        p[0].data = torch.zeros(8)

    def cut_where_it_lies(p, opt):
        p[0].data = p[0].data[:8]

    def state_of_another_size(p, opt):
        opt.m = [torch.zeros(63), opt.m[1]]

    def state_of_another_type(p, opt):
        opt.v = [opt.v[0], torch.zeros(64, dtype=torch.float64)]

    def state_gone(p, opt):
        opt.v = [opt.v[0], None]

    def another_type(p, opt):
        p[1].data = torch.zeros(64, dtype=torch.float16)

    def strided(p, opt):
        p[1].data = torch.zeros(128)[::2]

    def list_too_short(p, opt):
        opt.m = opt.m[:1]

    def master_of_fp32(p, opt):
        opt.master = [torch.zeros(64), None]

    def one_more(p, opt):
        opt.params.append(torch.zeros(64))

    for change in (replaced_by_a_shorter_one, cut_where_it_lies, state_of_another_size, state_of_another_type, state_gone, another_type, strided,
                   list_too_short, master_of_fp32, one_more):
        p, opt = fresh()
        change(p, opt)
        calls = len(lib.calls)
        for _ in range(2):                                                  # and again: nothing of the change has stuck
            with pytest.raises(binding.CpmtpError):
                opt.step([torch.zeros(64)] * len(opt.params), 2, lr=0.1)
                pytest.fail(f"{change.__name__} was accepted")
        assert len(lib.calls) == calls
    with pytest.raises(binding.CpmtpError):
        opt.m = [1, 2]


def test_nothing_changed_means_nothing_is_written_anew(lib, monkeypatch):
    p = torch.zeros(64)
    opt = binding.AdamW([p])
    monkeypatch.setattr(opt, "_bind", lambda: pytest.fail("the descriptors were written anew"))
    for t in range(1, 4):
        p.add_(1)
        opt.step([torch.zeros(64)], t, lr=0.1)


def test_memory_that_two_tensors_share_is_refused(lib):
    """The tensors of a step are updated at the same time, in no order."""
    flat, other = torch.zeros(600), torch.zeros(300)
    half = [flat[:300], flat[300:]]
    binding.AdamW(half)                                                     # next to one another is fine
    states = dict(m=[torch.zeros(300) for _ in range(2)], v=[torch.zeros(300) for _ in range(2)])
    binding.AdamW(half, state=states)
    bad = [dict(params=[flat, flat]), dict(params=[flat[:300], flat[299:]]), dict(params=[flat[:300], flat[10:20], other]),
           dict(params=half, state=dict(states, m=[other, other])), dict(params=half, state=dict(m=states["m"], v=states["m"])),
           dict(params=half, state=dict(states, v=[other, flat[:300]])),
           dict(params=[flat[:300].to(torch.bfloat16), flat[300:].to(torch.bfloat16)], master=[other, other])]
    for i, kw in enumerate(bad):
        with pytest.raises(binding.CpmtpError):
            binding.AdamW(kw.pop("params"), **kw)
            pytest.fail(f"case {i} was accepted")
    empty = [torch.zeros(0), torch.zeros(0), flat]
    binding.AdamW(empty)
    opt = binding.AdamW(half)
    half[1].data = flat[1:301]
    with pytest.raises(binding.CpmtpError):
        opt.step([torch.zeros(300)] * 2, 1, lr=0.1)
    assert not lib.calls


def test_a_state_is_given_as_a_whole(lib):
    """8-bit codes without their exponents, or one moment without the other, are the states of no run."""
    p = torch.zeros(600)
    full = {32: dict(m=[torch.zeros(600)], v=[torch.zeros(600)]),
            8: dict(m=[torch.zeros(600, dtype=torch.uint8)], v=[torch.zeros(600, dtype=torch.uint8)], m_exp=[torch.zeros(3, dtype=torch.uint8)],
                    v_exp=[torch.zeros(3, dtype=torch.uint8)])}
    for bits, state in full.items():
        binding.AdamW([p], bits=bits, state=state)
        binding.AdamW([p], bits=bits, state=dict.fromkeys(state))           # (None for all: a new run)
        for name in state:
            for less in ({k: t for k, t in state.items() if k != name}, dict(state, **{name: None})):
                with pytest.raises(binding.CpmtpError):
                    binding.AdamW([p], bits=bits, state=less)
                    pytest.fail(f"{bits} bits without {name} were accepted")
    binding.AdamW([p], state=dict(full[32], m_exp=None, v_exp=None))


@pytest.mark.parametrize("missing", [(), (0,), (4,), (1, 2), (0, 1, 2, 3, 4)])
@pytest.mark.parametrize("mixed", [False, True])
def test_missing_gradients_leave_their_places_empty(lib, missing, mixed):
    sizes = [3, 300, 0, 17, 256]
    opt = binding.AdamW([torch.zeros(n) for n in sizes])
    for t in (1, 2):                                                        # (a second time: what the first one wrote is there)
        grads = [None if i in missing and t == 2 else torch.zeros(n, dtype=torch.bfloat16 if mixed and i % 2 else torch.float32)
                 for i, n in enumerate(sizes)]
        opt.step(grads, t, lr=0.1)
        check(lib, opt, grads)
        for got, g in zip(lib.last, grads):
            assert g is None or got["grad_type"] == binding._TYPES[g.dtype]
    table = binding._Descriptors(len(sizes))
    table.put_grads(grads, -1)
    got = (binding.CAdamWTensor * len(sizes)).from_address(table.address)
    assert [t.numel for t in got] == [0 if g is None else g.numel() for g in grads]


def test_one_missing_gradient_costs_no_more_than_its_place():
    """The time of a call grows with the number of tensors, whether a gradient is missing or not: it was 50 times that of a full list
    at 300 tensors; the two are within half of one another now, and three times leaves room for a busy machine."""
    n = 600
    full = [torch.zeros(4) for _ in range(n)]
    holed = [None if i == n // 2 else g for i, g in enumerate(full)]
    table = binding._Descriptors(n)

    def best(grads):
        times = []
        for _ in range(15):
            start = time.perf_counter()
            table.put_grads(grads, -1)
            times.append(time.perf_counter() - start)
        return min(times)

    assert best(holed) < 3 * best(full)


def test_the_clocks_layout_and_checks():
    import os
    import re

    from paper_2410_17765_b200 import build

    build.build()
    lib = binding.load_library()
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "cpmtp.h")).read()
    body = re.search(r"typedef struct cpmtp_adamw_clock \{(.*?)\}", header, re.S).group(1)
    body = re.sub(r"/\*.*?\*/", "", body, flags=re.S)
    assert [d.split()[-1] for d in body.split(";") if d.strip()] == [f[0] for f in binding.CAdamWClock._fields_]
    clock = binding.StepClock(0.25, step=41, seed=-1, device="cpu")
    assert int(clock.step) == 41 and float(clock.lr) == 0.25 and clock.block.numel() == ctypes.sizeof(binding.CAdamWClock) == 40
    clock.lr.fill_(0.5)
    assert binding.CAdamWClock.from_buffer_copy(bytes(clock.block.tolist())).lr == 0.5
    assert binding.CAdamWClock.from_buffer_copy(bytes(clock.block.tolist())).seed == 0xFFFFFFFF
    hyper = binding.CAdamWHyper(0.1, 0.9, 0.95, 1e-8, 0.1, 1, 0, 32, None)
    at = ctypes.c_void_p(4096)
    assert lib.cpmtp_adamw_step_clocked(None, 0, ctypes.byref(hyper), None, None) == -1
    assert lib.cpmtp_adamw_step_clocked(None, 0, None, at, None) == -1
    assert lib.cpmtp_adamw_step_clocked(None, 0, ctypes.byref(hyper), ctypes.c_void_p(4100), None) == -3
    assert lib.cpmtp_adamw_step_clocked(None, 1, ctypes.byref(hyper), at, None) == -1
    hyper.beta1 = 1.0
    assert lib.cpmtp_adamw_step_clocked(None, 0, ctypes.byref(hyper), at, None) == -2
