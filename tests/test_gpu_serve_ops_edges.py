"""Graphs, streams, shared workspaces, long offsets and give-ups of the serving operators."""
import numpy as np
import pytest
import torch

from test_gpu_cache import Case, check_attend, check_evict

pytestmark = pytest.mark.gpu


def test_attend_and_append_replay_from_a_graph():
    """A captured step follows its inputs: lengths, tables, queries and cache contents change between replays."""
    from paper_2410_17765_b200 import binding

    c = Case([600, 130, 64], 2, 64, 16, Q=3, Hq=4, seed=1)
    k = torch.randn(3, 3, 2, 64, device="cuda").to(torch.bfloat16)
    cache, out = c.cache(), {}

    def step():
        binding.cache_append(cache, k, k, c.table, c.lens_t, dev_status=c.status)
        return binding.cache_attend(cache, c.q, c.table, c.lens_t, out=out, want_lse=True, workspace=ws, dev_status=c.status)

    ws = binding.alloc_workspace(binding.cache_attend_workspace_bytes(cache, 3, c.table.shape[1], 3, 4))
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([600, 130, 64], [599, 3, 20], [300, 128, 1]):
        c.lens_t.copy_(torch.tensor(lens, dtype=torch.int32))
        c.q.normal_()
        k.normal_()
        before = c.acc.clone()
        graph.replay()
        got = {n: t.clone() for n, t in out.items()}
        acc = c.acc.clone()
        c.acc.copy_(before)
        want = step()
        torch.cuda.synchronize()
        assert torch.equal(got["out"], want["out"]) and torch.equal(got["lse"], want["lse"])
        assert torch.equal(torch.nan_to_num(acc, 9.0), torch.nan_to_num(c.acc, 9.0))
        c.status.zero_()


def test_two_graphs_share_a_workspace():
    from paper_2410_17765_b200 import binding

    cases = [Case([900, 33], 2, 128, 64, Hq=8, seed=2), Case([400, 401], 2, 128, 64, Hq=8, seed=3)]
    sizes = [binding.cache_attend_workspace_bytes(c.cache(), 2, c.table.shape[1], 1, 8) for c in cases]
    ws = binding.alloc_workspace(max(sizes))
    want = [binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=False)["out"] for c in cases]
    graphs, outs = [], []
    for c in cases:
        cache, out = c.cache(), {}
        binding.cache_attend(cache, c.q, c.table, c.lens_t, accumulate=False, out=out, workspace=ws)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.cache_attend(cache, c.q, c.table, c.lens_t, accumulate=False, out=out, workspace=ws)
        graphs.append((g, cache))
        outs.append(out["out"])
    for _ in range(3):
        ws.fill_(255)
        for o in outs:
            o.zero_()
        for g, _ in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


def test_workspaces_may_hold_anything():
    from paper_2410_17765_b200 import binding

    c = Case([900, 33, 2000], 2, 64, 64, Hq=8, seed=2)
    n = binding.cache_attend_workspace_bytes(c.cache(), 3, c.table.shape[1], 1, 8)
    first = None
    for fill in (0, 255, 127):
        acc = c.acc.clone()
        out = binding.cache_attend(binding.PagedCache(c.k, c.v, acc), c.q, c.table, c.lens_t, workspace=torch.full((n,), fill, dtype=torch.uint8, device="cuda"))["out"]
        if first is None:
            first = (out, acc)
        assert torch.equal(out, first[0]) and torch.equal(torch.nan_to_num(acc, 9.0), torch.nan_to_num(first[1], 9.0))


def test_evict_and_sample_replay_from_a_graph():
    from paper_2410_17765_b200 import binding

    c = Case([500, 90, 300], 2, 16, 16, more=4, seed=6)
    cache, out, drawn = c.cache(), {}, {}
    x, u = torch.randn(5, 3001, device="cuda"), torch.rand(5, device="cuda")
    T = torch.full((5,), 0.7, device="cuda")

    def step():
        binding.cache_evict(cache, c.table, c.lens_t, c.table_out, 64, recent=9, out=out)
        binding.sample_logits(x, u, temperature=T, top_k=40, top_p=0.9, want_kept=True, out=drawn)

    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(3):
        c.acc.uniform_()
        x.normal_()
        u.uniform_()
        T.uniform_()
        g.replay()
        got = [t.clone() for t in (*out.values(), *drawn.values())]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (*out.values(), *drawn.values())))


def test_other_streams():
    from paper_2410_17765_b200 import binding

    side = torch.cuda.Stream()
    c = Case([700, 130], 2, 64, 16, Hq=4, more=8, seed=8)
    x, u = torch.randn(7, 5000, device="cuda"), torch.rand(7, device="cuda")
    want = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=False)["out"], binding.sample_logits(x, u, top_p=0.8)["tokens"]
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=False)["out"], binding.sample_logits(x, u, top_p=0.8)["tokens"]
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    with torch.cuda.stream(side):
        check_evict(c, 100, 5)


def test_two_calls_at_once():
    """Two streams, each with its own workspace and outputs, many calls in flight."""
    from paper_2410_17765_b200 import binding

    cases = [Case([3000, 700], 2, 64, 64, Hq=8, acc=False, seed=s) for s in (1, 2)]
    want = [binding.cache_attend(c.cache(), c.q, c.table, c.lens_t)["out"].clone() for c in cases]
    x, u = torch.randn(40, 9000, device="cuda"), torch.rand(40, device="cuda")
    tokens = binding.sample_logits(x, u, top_p=0.9)["tokens"]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(3)]
    got = [[], [], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(binding.cache_attend(cases[i].cache(), cases[i].q, cases[i].table, cases[i].lens_t)["out"])
        with torch.cuda.stream(streams[2]):
            got[2].append(binding.sample_logits(x, u, top_p=0.9)["tokens"])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])
    assert all(torch.equal(o, tokens) for o in got[2])


def test_offsets_beyond_32_bits():
    """A cache of more than 2^32 bytes, and of more than 2^31 elements, with the sequence in its last pages."""
    from paper_2410_17765_b200 import binding

    H, D, page = 8, 128, 64
    P = (1 << 31) // (H * D * page) + 40
    big = torch.empty(P, page, H, D, dtype=torch.bfloat16, device="cuda")
    small = Case([150], H, D, page, Hq=16, Q=2, more=3, seed=11)
    pages = [P - 1 - 2 * i for i in range(small.table.shape[1])]
    table = torch.tensor([pages], dtype=torch.int32, device="cuda")
    acc = torch.zeros(P, H, page, device="cuda")
    cache = binding.PagedCache(big, big, acc)
    k = small.k[small.table[0, :3].long()].reshape(1, 3 * page, H, D)[:, :150]
    binding.cache_append(cache, k, k, table, small.lens_t, dev_status=small.status)
    got = binding.cache_attend(cache, small.q, table, small.lens_t)["out"]
    want = binding.cache_attend(binding.PagedCache(small.k, small.k), small.q, small.table, small.lens_t)["out"]
    assert int(small.status.item()) == 0 and torch.equal(got, want)
    out = torch.tensor([[P - 2, P - 4]], dtype=torch.int32, device="cuda")
    kept = binding.cache_evict(cache, table, small.lens_t, out, 100, recent=10, dev_status=small.status)["kept"]
    assert int(small.status.item()) == 0
    for h in range(H):
        slots = kept[0, h].long()
        moved = big[out[0].long()][:, :, h].reshape(-1, D)[:100]
        assert torch.equal(moved, big[table[0].long()][:, :, h].reshape(-1, D)[slots])


def test_sizes_of_nothing():
    from paper_2410_17765_b200 import binding

    c = Case([30, 20], 2, 64, 16, more=4)
    cache, i32 = c.cache(), dict(dtype=torch.int32, device="cuda")
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    assert binding.cache_attend(cache, c.q[:0], c.table[:0], none)["out"].shape == (0, 1, 2, 64)
    assert binding.cache_attend(cache, c.q[:, :0], c.table, c.lens_t)["out"].shape == (2, 0, 2, 64)
    binding.cache_append(cache, c.q[:0], c.q[:0], c.table[:0], none)
    assert binding.cache_evict(cache, c.table[:0], none, c.table_out[:0], 10)["lens"].numel() == 0
    r = binding.cache_attend(cache, c.q, torch.empty(2, 0, **i32), torch.zeros(2, **i32), want_lse=True)
    assert (r["out"] == 0).all() and torch.isneginf(r["lse"]).all()
    assert binding.sample_logits(torch.empty(0, 10, device="cuda"), torch.empty(0, device="cuda"))["tokens"].numel() == 0


def test_same_page_in_two_sequences_for_reading():
    """A prefix that two sequences share, without weights."""
    from paper_2410_17765_b200 import binding

    c = Case([200, 200], 2, 64, 16, Hq=4, acc=False)
    t = c.table.clone()
    t[1, :8] = t[0, :8]
    c.table_np[:] = t.cpu().numpy()
    c.table = t
    check_attend(c)


@pytest.mark.parametrize("skip", [1, 2, 3])
def test_bounded_waits_give_up_and_the_library_stays_usable(skip):
    """A load that never comes (left out by the test hook): the kernel gives up after the limit and says so; the next call is right."""
    from paper_2410_17765_b200 import binding

    c = Case([1500, 700], 2, 64, 64, Hq=4, seed=5)
    want = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=False)["out"]
    torch.cuda.synchronize()
    with binding.knobs(CPMTP_WAIT_LIMIT_US=20000, CPMTP_TEST_SKIP_LOAD=skip):
        binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=False, dev_status=c.status)
        torch.cuda.synchronize()
    # (a third load is one of a second tile, which only some shares have)
    assert int(c.status.item()) == 2 or skip == 3
    c.status.zero_()
    got = binding.cache_attend(c.cache(), c.q, c.table, c.lens_t, accumulate=False, dev_status=c.status)["out"]
    assert int(c.status.item()) == 0 and torch.equal(got, want)


def test_refusals_of_the_binding():
    from paper_2410_17765_b200 import binding

    c = Case([30, 20], 2, 64, 16, Hq=4, more=4)
    cache = c.cache()
    bad = binding.CpmtpError
    for args in ((c.q.float(), c.table, c.lens_t), (c.q[:, :, :3], c.table, c.lens_t), (c.q, c.table.long(), c.lens_t), (c.q, c.table[:1], c.lens_t),
                 (c.q, c.table, c.lens_t.long()), (c.q, c.table, c.lens_t[:1]), (c.q.cpu(), c.table, c.lens_t), (c.q, c.table.cpu(), c.lens_t)):
        with pytest.raises(bad):
            binding.cache_attend(cache, *args)
    for kw in (dict(q_lens=c.lens_t.long()), dict(out=dict(out=c.q.float())), dict(out=dict(lse=torch.zeros(2, 1, 4, device="cuda").double())),
               dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda")), dict(workspace=torch.empty(1 << 20, device="cuda")), dict(scale=float("nan")),
               dict(out=dict(out=c.q[:, :, :1].expand(2, 1, 4, 64)))):
        with pytest.raises(bad):
            binding.cache_attend(cache, c.q, c.table, c.lens_t, **kw)
    for kw in (dict(budget=0), dict(budget=10, recent=11), dict(budget=10, recent=-1), dict(budget=1000)):
        with pytest.raises(bad):
            binding.cache_evict(cache, c.table, c.lens_t, c.table_out, **kw)
    with pytest.raises(bad):
        binding.cache_evict(binding.PagedCache(c.k, c.v), c.table, c.lens_t, c.table_out, 10)
    with pytest.raises(bad):
        binding.cache_evict(cache, c.table, c.lens_t, c.table_out, 10, out=dict(lens=c.lens_t))
    with pytest.raises(bad):
        binding.cache_append(cache, c.q, c.q, c.table, c.lens_t)          # four heads into a cache of two
    x, u = torch.randn(2, 50, device="cuda"), torch.rand(2, device="cuda")
    for args in ((x.half(), u), (x.t(), u), (x, u[:1]), (x, u.double()), (x.cpu(), u)):
        with pytest.raises(bad):
            binding.sample_logits(*args)
    for kw in (dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(top_k=-1), dict(top_p=-0.1), dict(min_p=-0.1),
               dict(top_p=u.double()), dict(top_k=u), dict(temperature=u[:1]), dict(given=u), dict(given=torch.zeros(3, dtype=torch.int32, device="cuda"))):
        with pytest.raises(bad):
            binding.sample_logits(x, u, **kw)
