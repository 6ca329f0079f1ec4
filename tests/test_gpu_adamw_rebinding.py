"""An optimiser whose tensors are given other memory between steps goes on as one that was made with them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("master", [False, True])
def test_replaced_parameters_and_states(bits, master):
    from paper_2410_17765_b200 import binding

    sizes = [700, 256, 5000]
    gen = torch.Generator(device="cuda").manual_seed(2)

    def draw(n):
        return torch.randn(n, generator=gen, device="cuda").to(torch.bfloat16)

    start = [draw(n) for n in sizes]
    a, b = (binding.AdamW([p.clone() for p in start], bits=bits, master=master) for _ in range(2))
    names = ["m", "v"] + (["m_exp", "v_exp"] if bits == 8 else []) + (["master"] if master else [])
    for t in range(1, 6):
        grads = [draw(n) for n in sizes]
        a.step(grads, t, lr=0.01, seed=4)
        b.step(grads, t, lr=0.01, seed=4)
        for i in range(3):
            assert torch.equal(a.params[i], b.params[i])
            for k in names:
                assert torch.equal(getattr(a, k)[i], getattr(b, k)[i]), (t, i, k)
        old = [b.params[t % 3].data]
        b.params[t % 3].data = b.params[t % 3].data.clone()                 # as a module's .to() does
        for k in names:
            old += getattr(b, k)
            setattr(b, k, [x.clone() for x in getattr(b, k)])               # as a restored checkpoint does
        before = [x.clone() for x in old]
        b.step([torch.zeros_like(p) for p in b.params], t, lr=0.0, seed=4)
        a.step([torch.zeros_like(p) for p in a.params], t, lr=0.0, seed=4)
        assert all(torch.equal(x, y) for x, y in zip(old, before))          # what was replaced is left alone
