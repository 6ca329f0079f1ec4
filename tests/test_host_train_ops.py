"""CPU-only checks of the training-step entry points: sizes of workspaces, structure layouts, and that bad arguments are
rejected before a GPU is touched."""
import ctypes
import os
import re

import pytest
import torch

from paper_2410_17765_b200 import binding, build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = ctypes.c_void_p(4096)                                # an aligned address that no accepted call would be given here
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
            words = decl.replace("*", " ").split()
            if not words:
                continue
            rows = words[0] == "cpmtp_rows"
            for n in " ".join(words[1:] if words[0] != "const" else words[2:]).split(","):
                out += [n.strip(), "ld_" + n.strip()] if rows else [n.strip()]
        return out

    for struct, cls in (("cpmtp_embed_shape", binding.CEmbedShape), ("cpmtp_norm_args", binding.CNormArgs),
                        ("cpmtp_adamw_tensor", binding.CAdamWTensor), ("cpmtp_adamw_hyper", binding.CAdamWHyper)):
        assert names(struct) == [f[0] for f in cls._fields_], struct
    assert re.search(r"#define CPMTP_ADAMW_BLOCK (\d+)", header).group(1) == str(binding.ADAMW_BLOCK)


def embed(**kw):
    a = dict(T=8, V=100, d=16, type=binding.BF16, ld_table=16, ld_rows=16, scale=1.0, flags=0)
    a.update(kw)
    return binding.CEmbedShape(*[a[f[0]] for f in binding.CEmbedShape._fields_])


@pytest.mark.parametrize("bad", [dict(T=-1), dict(T=1 << 30), dict(V=0), dict(V=-5), dict(V=1 << 30), dict(d=0), dict(d=1 << 24), dict(type=2),
                                 dict(ld_table=15), dict(ld_rows=15)])
def test_embed_shapes_are_checked(lib, bad):
    s = embed(**bad)
    assert lib.cpmtp_embed_workspace_bytes(ctypes.byref(s)) == 0
    assert lib.cpmtp_embed_forward(ctypes.byref(s), P, P, P, None, None) == -2
    assert lib.cpmtp_embed_backward(ctypes.byref(s), P, P, P, P, 1 << 20, None, None) == -2


def test_embed_arguments_are_checked(lib):
    s = embed()
    need = lib.cpmtp_embed_workspace_bytes(ctypes.byref(s))
    assert need >= 2 * 8 * 8
    odd = ctypes.c_void_p(4097)
    assert lib.cpmtp_embed_forward(None, P, P, P, None, None) == -1
    for args in ((None, P, P), (P, None, P), (P, P, None)):
        assert lib.cpmtp_embed_forward(ctypes.byref(s), *args, None, None) == -1
    for args in ((odd, P, P), (P, odd, P), (P, P, odd)):
        assert lib.cpmtp_embed_forward(ctypes.byref(s), *args, None, None) == -3
    assert lib.cpmtp_embed_backward(ctypes.byref(s), P, P, P, None, need, None, None) == -1
    assert lib.cpmtp_embed_backward(ctypes.byref(s), P, P, P, ctypes.c_void_p(4096 + 16), need, None, None) == -3
    assert lib.cpmtp_embed_backward(ctypes.byref(s), P, P, P, P, need - 1, None, None) == -4
    many = embed(T=(1 << 24) + 1)                        # the lookup takes them, the gradient's sort does not
    assert lib.cpmtp_embed_workspace_bytes(ctypes.byref(many)) == 0
    assert lib.cpmtp_embed_backward(ctypes.byref(many), P, P, P, P, 1 << 40, None, None) == -7
    none = embed(T=0, flags=binding.FLAG_ACCUM_GRADS)
    assert lib.cpmtp_embed_forward(ctypes.byref(none), None, None, None, None, None) == 0
    assert lib.cpmtp_embed_backward(ctypes.byref(none), None, None, None, None, 0, None, None) == 0
    # many chunks keep two partial rows each; more key bits than two passes of the sort hold make three
    assert lib.cpmtp_embed_workspace_bytes(ctypes.byref(embed(T=6400))) >= 2 * 200 * 256 * 4 + 2 * 8 * 6400
    assert lib.cpmtp_embed_workspace_bytes(ctypes.byref(embed(V=(1 << 30) - 1))) > 0


def norm(**kw):
    a = binding.CNormArgs()
    base = dict(N=4, d=32, stream_type=binding.BF16, gate_kind=binding.GATE_CHANNEL, eps=1e-6, res_scale=1.0, w_post=4096, w_pre=4096, rstd_post=4096,
                rstd_pre=4096, dw_post=4096, dw_pre=4096)
    for n in ("x", "block", "gate", "x_out", "y", "dy", "dx_out", "dx", "dblock", "dgate"):
        base[n], base["ld_" + n] = 4096, 32
    base.update(kw)
    for k, v in base.items():
        setattr(a, k, v)
    return a


FORWARD_BAD = [(dict(N=-1), -2), (dict(d=0), -2), (dict(d=8193), -7), (dict(stream_type=3), -2), (dict(gate_kind=3), -2), (dict(eps=0.0), -2),
               (dict(eps=float("nan")), -2), (dict(res_scale=float("inf")), -2), (dict(x=None), -1), (dict(ld_x=31), -2), (dict(x=4097), -3),
               (dict(block=None), -2), (dict(gate=None), -1), (dict(ld_gate=31), -2), (dict(x_out=None), -1), (dict(y=None), -1), (dict(ld_y=0), -2),
               (dict(block=4097), -3), (dict(w_pre=4097), -3), (dict(rstd_pre=4098), -3),
               (dict(block=None, gate_kind=0, w_post=None, res_scale=0.5), -2), (dict(block=None, gate_kind=0, w_post=None, w_pre=None), -1)]
BACKWARD_BAD = [(dict(N=-1), -2), (dict(d=8193), -7), (dict(x_out=None), -1), (dict(dy=None), -1), (dict(dy=None, dw_pre=None, dx_out=None), -1),
                (dict(w_pre=None), -1), (dict(rstd_pre=None), -1), (dict(rstd_post=None), -1), (dict(w_post=None), -1), (dict(ld_dy=31), -2),
                (dict(dx=4097), -3), (dict(ld_dblock=31), -2), (dict(dgate=4097), -3), (dict(gate_kind=0), -1), (dict(dw_pre=4097), -3),
                (dict(dx=None, dblock=None, dgate=None, dw_post=None, dw_pre=None), -1)]


@pytest.mark.parametrize("bad,code", FORWARD_BAD)
def test_norm_forward_arguments_are_checked(lib, bad, code):
    assert lib.cpmtp_norm_forward(ctypes.byref(norm(**bad)), None) == code


@pytest.mark.parametrize("bad,code", BACKWARD_BAD)
def test_norm_backward_arguments_are_checked(lib, bad, code):
    assert lib.cpmtp_norm_backward(ctypes.byref(norm(**bad)), P, 1 << 20, None) == code


def test_norm_workspace_and_empty_calls(lib):
    a = norm()
    need = lib.cpmtp_norm_workspace_bytes(ctypes.byref(a))
    assert need >= 2 * 4 * 32
    assert lib.cpmtp_norm_backward(ctypes.byref(a), ctypes.c_void_p(4104), need, None) == -3
    if NO_GPU:                                           # the workspace is looked at after the device
        assert lib.cpmtp_norm_backward(ctypes.byref(a), P, need, None) < 0
    assert lib.cpmtp_norm_forward(None, None) == -1
    assert lib.cpmtp_norm_forward(ctypes.byref(norm(N=0, x=None, block=None, y=None)), None) == 0
    assert lib.cpmtp_norm_backward(ctypes.byref(norm(N=0, dw_post=None, dw_pre=None)), None, 0, None) == 0


def adamw(**kw):
    a = dict(param=4096, grad=4096, master=None, m=4096, v=4096, m_exp=4096, v_exp=4096, numel=10, param_type=binding.BF16, grad_type=binding.BF16,
             lr_scale=1.0, decay_scale=1.0)
    a.update(kw)
    return (binding.CAdamWTensor * 1)(binding.CAdamWTensor(*[a[f[0]] for f in binding.CAdamWTensor._fields_]))


def hyper(**kw):
    a = dict(lr=0.1, beta1=0.9, beta2=0.95, eps=1e-8, weight_decay=0.1, step=1, seed=0, state_bits=8, coef=None)
    a.update(kw)
    return binding.CAdamWHyper(*[a[f[0]] for f in binding.CAdamWHyper._fields_])


@pytest.mark.parametrize("bad,code", [(dict(numel=-1), -2), (dict(numel=1 << 40), -2), (dict(param_type=2), -2), (dict(grad_type=-1), -2),
                                      (dict(param=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(m_exp=None), -1), (dict(v_exp=None), -1),
                                      (dict(param=4097), -3), (dict(grad=4097), -3), (dict(master=4098), -3),
                                      (dict(master=4096, param_type=binding.F32), -2), (dict(lr_scale=float("nan")), -2),
                                      (dict(decay_scale=float("inf")), -2)])
def test_adamw_tensors_are_checked(lib, bad, code):
    assert lib.cpmtp_adamw_step(adamw(**bad), 1, ctypes.byref(hyper()), None) == code


@pytest.mark.parametrize("bad", [dict(lr=-1.0), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")),
                                 dict(eps=-1e-8), dict(weight_decay=float("nan")), dict(step=0), dict(state_bits=16)])
def test_adamw_hyperparameters_are_checked(lib, bad):
    assert lib.cpmtp_adamw_step(adamw(), 1, ctypes.byref(hyper(**bad)), None) == -2


def test_optimiser_edges(lib):
    assert lib.cpmtp_adamw_step(adamw(), 1, None, None) == -1
    assert lib.cpmtp_adamw_step(None, 1, ctypes.byref(hyper()), None) == -1
    assert lib.cpmtp_adamw_step(adamw(), -1, ctypes.byref(hyper()), None) == -2
    assert lib.cpmtp_adamw_step(adamw(m=4098), 1, ctypes.byref(hyper(state_bits=32)), None) == -3
    assert lib.cpmtp_adamw_step(adamw(), 1, ctypes.byref(hyper(coef=4097)), None) == -3
    need = lib.cpmtp_grad_norm_workspace_bytes(adamw(), 1)
    assert need > 0 and lib.cpmtp_grad_norm_workspace_bytes(adamw(numel=-1), 1) == 0
    assert lib.cpmtp_grad_norm(adamw(), 1, 0.0, P, P, P, need, None) == -2
    assert lib.cpmtp_grad_norm(adamw(), 1, 1.0, None, None, P, need, None) == -1
    assert lib.cpmtp_grad_norm(adamw(), 1, 1.0, P, P, None, need, None) == -1
    assert lib.cpmtp_grad_norm(adamw(), 1, 1.0, P, P, P, need - 1, None) == -4
    assert lib.cpmtp_adamw_state_values(P, P, -1, 0, P, None) == -2
    assert lib.cpmtp_adamw_state_values(None, P, 5, 0, P, None) == -1
    assert lib.cpmtp_adamw_state_values(None, None, 0, 0, None, None) == 0


def test_the_binding_refuses_cpu_tensors():
    E, x = torch.zeros(4, 8, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    for f in (lambda: binding.embed_forward(E, x), lambda: binding.embed_backward(E[:2], x, 4), lambda: binding.norm_forward(E, E[0]),
              lambda: binding.norm_backward(E, E, E[0], torch.zeros(4)), lambda: binding.AdamW([E]), lambda: binding.grad_norm([E])):
        with pytest.raises(binding.CpmtpError):
            f()
