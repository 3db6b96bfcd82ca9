"""Calls that the documentation of the decoding and distillation operators allows and that
are easily got wrong: odd strides of sizes of one, explicit streams, a workspace larger
than needed and full of anything, several calls in flight with workspaces of their own."""
import pytest
import torch

from test_gpu_distill import make as distill_inputs
from test_gpu_sample import logits
from test_gpu_window import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    from paper_2412_00408_amd import quake
    return quake


def test_strides_of_sizes_of_one_are_not_used(q):
    for skv in (1, 70):
        x = make(1, 1, skv, 1, 1, 64, torch.bfloat16, 41)
        want = q.quake_attention_window(*x, window=50)
        odd = [a.as_strided(a.shape, (3, a.stride(1) if a.shape[1] > 1 else 5, 7, 1)) for a in x]
        o = torch.zeros(64, dtype=torch.bfloat16, device="cuda").as_strided((1, 1, 1, 64), (1, 1, 1, 1))
        for ws in (None, q.attention_window_workspace(*x[:2], 50)):
            q.quake_attention_window(*odd, o, window=50, workspace=ws)
            assert torch.equal(o, want)


def calls(q):
    """(name, call, its inputs): what runs split or in chunks, with its own workspace."""
    x = make(1, 1, 9000, 8, 1, 128, torch.bfloat16, 42)
    l = logits(2, 80000, torch.float32, 43)
    d = distill_inputs(3, 60000, 40, torch.bfloat16, 44)
    u, p = torch.tensor([0.3, 0.8], device="cuda"), torch.tensor([0.9, 0.6], device="cuda")
    wx, wl, wd = q.attention_window_workspace(*x[:2], 9000), q.sample_workspace(l), q.distill_workspace(d[0])
    assert None not in (wx, wl, wd)
    return [("window", lambda ws=wx, **kw: [q.quake_attention_window(*x, window=9000, workspace=ws, **kw)], wx),
            ("sample", lambda ws=wl, **kw: list(q.quake_sample(l, u, top_p=p, workspace=ws, **kw)), wl),
            ("plain", lambda ws=wl, **kw: list(q.quake_sample(l, u, workspace=ws, **kw)), wl),
            ("distill", lambda ws=wd, **kw: list(q.quake_distill(d[0], d[1], d[2], weight=d[3], grad=True,
                                                                 workspace=ws, **kw)), wd)]


def test_larger_workspaces_full_of_anything(q):
    for name, call, ws in calls(q):
        want = call()
        for fill in (0, 0x7F, 0xFF):
            big = torch.full((ws.numel() + 4096,), fill, dtype=torch.uint8, device="cuda")
            got = call(ws=big)
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (name, fill)
            assert (big[ws.numel():] == fill).all()          # nothing behind its size is written
            got = call(ws=big[16:])
            assert all(torch.equal(a, b) for a, b in zip(got, want)), (name, fill)


def test_several_calls_in_flight(q):
    for name, call, ws in calls(q):
        want = call()
        streams = [torch.cuda.Stream() for _ in range(3)]
        spaces = [torch.empty_like(ws) for _ in streams]
        torch.cuda.synchronize()
        got = []
        for _ in range(4):
            for s, w in zip(streams, spaces):
                got.append(call(ws=w, stream=s))             # the binding's own argument
        torch.cuda.synchronize()
        for g in got:
            assert all(torch.equal(a, b) for a, b in zip(g, want)), name


def test_two_graphs_one_after_the_other_share_a_workspace(q):
    for name, call, ws in calls(q):
        want = call()
        graphs, outs = [], []
        torch.cuda.synchronize()
        for _ in range(2):
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                outs.append(call())
            graphs.append(g)
        for _ in range(3):
            for g, o in zip(graphs, outs):
                for t in o:
                    t.zero_()
                g.replay()
                torch.cuda.synchronize()
                assert all(torch.equal(a, b) for a, b in zip(o, want)), name
