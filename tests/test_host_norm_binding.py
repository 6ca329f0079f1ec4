"""CPU-only checks of what the binding's norms do with the dictionaries they are given: a stand-in for the library takes the calls."""
import pytest
import torch

from paper_2410_17765_b200 import binding


class Nothing:
    """In the library's place: keeps each call's arguments and does nothing."""

    def __init__(self):
        self.args = None

    def keep(self, args):
        self.args = {f[0]: getattr(args._obj, f[0]) for f in args._obj._fields_}

    def cpmtp_norm_forward(self, args, stream):
        self.keep(args)
        return 0

    def cpmtp_norm_workspace_bytes(self, args):
        return 256

    def cpmtp_norm_backward(self, args, workspace, size, stream):
        self.keep(args)
        return 0


@pytest.fixture
def lib(monkeypatch):
    fake = Nothing()
    monkeypatch.setattr(binding, "load_library", lambda: fake)
    monkeypatch.setattr(binding, "_device", lambda t: t.get_device())
    monkeypatch.setattr(binding, "_raw_stream", lambda dev: 0)
    monkeypatch.setattr(binding, "alloc_workspace", lambda n, device: torch.empty(n, dtype=torch.uint8))
    return fake


N, D = 4, 32


def rows():
    return torch.zeros(N, D, dtype=torch.bfloat16)


def test_forward_leaves_the_dictionary_as_it_is(lib):
    x, w, block = rows(), torch.ones(D, dtype=torch.bfloat16), rows()
    out = dict(y=rows())
    r = binding.norm_forward(x, w, out=out)
    assert list(out) == ["y"] and r["y"] is out["y"] and r["x_out"] is x and r["rstd_post"] is None
    # the same dictionary in a call with a block: x is not written to
    r = binding.norm_forward(x, w, block=block, w_post=w, out=out)
    assert r["x_out"] is not x and lib.args["x_out"] == r["x_out"].data_ptr() != x.data_ptr()
    assert list(out) == ["y"] and lib.args["y"] == out["y"].data_ptr()
    full = dict(x_out=x, y=rows(), rstd_pre=torch.zeros(N), rstd_post=torch.zeros(N))
    r = binding.norm_forward(x, w, block=block, w_post=w, out=dict(full))
    assert all(r[k] is t and lib.args[k] == t.data_ptr() for k, t in full.items())


def test_backward_leaves_the_dictionary_as_it_is(lib):
    x, w, dy, block, gate, rstd = rows(), torch.ones(D, dtype=torch.bfloat16), rows(), rows(), rows(), torch.ones(N)
    full = dict(dx=rows(), dblock=rows(), dgate=rows(), dw_post=torch.ones(D, dtype=torch.bfloat16), dw_pre=torch.ones(D, dtype=torch.bfloat16))
    out = dict(full)
    kw = dict(block=block, gate=gate, w_post=w, rstd_post=rstd)
    r = binding.norm_backward(dy, x, w, rstd, out=out, skip=("dx", "dw_post", "dgate"), **kw)
    assert all(out[k] is t for k, t in full.items()) and r["dx"] is None and r["dw_post"] is None and r["dgate"] is None
    assert r["dblock"] is full["dblock"] and r["dw_pre"] is full["dw_pre"]
    r = binding.norm_backward(dy, x, w, rstd, out=out)             # a norm alone: the block's gradients stay where they are
    assert all(out[k] is t for k, t in full.items()) and r["dblock"] is None and r["dx"] is full["dx"]
    r = binding.norm_backward(dy, x, w, rstd, out=out, accumulate=True, **kw)
    assert all(r[k] is t and lib.args[k] == t.data_ptr() for k, t in full.items()) and lib.args["flags"] == binding.FLAG_ACCUM_GRADS
    empty = {}
    r = binding.norm_backward(dy, x, w, rstd, out=empty, **kw)
    assert not empty and all(lib.args[k] == r[k].data_ptr() for k in full)


def test_eps_has_to_be_a_normal_number():
    """The rstd of a row of zeros would have an infinite square, and the gradient of that row be NaN."""
    import ctypes

    from paper_2410_17765_b200 import build

    build.build()
    args = binding.CNormArgs(0, D, binding.BF16, binding.GATE_NONE, 0, 2.0 ** -126, 1.0)       # (no rows: nothing is enqueued)
    args.w_pre = 4096
    real = binding.load_library()
    assert real.cpmtp_norm_forward(ctypes.byref(args), None) == 0
    for eps in (1e-40, 2.0 ** -127, 0.0, -1.0):
        args.eps = eps
        assert real.cpmtp_norm_forward(ctypes.byref(args), None) == -2
        assert real.cpmtp_norm_backward(ctypes.byref(args), None, 0, None) == -2
        assert real.cpmtp_norm_workspace_bytes(ctypes.byref(args)) == 0
