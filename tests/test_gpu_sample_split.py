"""quake_sample's rows split over workgroups (65536 words and more, up to 64 rows,
without a top-k) on the inputs, layouts and parameters that go wrong most easily, in
graphs and on streams, and EXACT's filters in both forms."""
import math

import numpy as np
import pytest
import torch

import ref64
from gpu_util import say
from test_gpu_sample import DTS, dev, logits, run

pytestmark = pytest.mark.gpu
COLS = 70001


@pytest.fixture(scope="module")
def q():
    from paper_2412_00408_amd import quake
    return quake


def test_which_rows_are_split(q):
    size = "quake_sample_workspace_size"
    assert q._size(size, 1, COLS) > 0 and q._size(size, 64, 65536) > 0
    assert q._size(size, 65, COLS) == 0 and q._size(size, 64, 65535) == 0


@pytest.mark.parametrize("dt", DTS, ids=["f32", "bf16", "f16"])
def test_masked_words_infinities_and_nan(q, dt):
    inf, nan = math.inf, math.nan
    x = logits(9, COLS, dt, 51)
    x[0] = -inf                                  # nothing allowed
    x[1, 1:] = -inf                              # one word, the first
    x[2, :-1] = -inf                             # the last
    x[3, ::2] = -inf
    x[4, 5] = nan
    x[4, 30000:60000] = nan
    x[5, 9] = inf                                # certain
    x[5, 60021] = inf
    x[6] = torch.finfo(dt).min                   # the type's lowest value everywhere
    x[7] = nan
    x[8, 1000:] = torch.finfo(dt).min            # as a mask
    u = [0.5, 0.5, 0.5, 0.25, 0.999, 0.75, 0.4, 0.5, 0.9]
    run(q, "split masked", x, u)
    run(q, "split masked top-p", x, u, top_p=[0.8] * 9)
    run(q, "split masked min-p", x, u, min_p=[0.01] * 9, temperature=[0.6] * 9)
    run(q, "split masked both", x, u, top_p=[0.95, 0.0, 1.0, 0.3] * 2 + [0.7], min_p=[0.01] * 9)
    run(q, "split masked greedy", x, u, temperature=[0.0] * 9)
    run(q, "split masked some greedy", x, u, temperature=[0.0, 1.0, 0.0] * 3, top_p=[0.9] * 9)


def test_equal_and_almost_equal_words(q):
    # every word in one bin of the weights: more candidates than a workgroup ranks
    for dt in (torch.float32, torch.bfloat16):
        x = torch.full((4, COLS), 1.25, dtype=dt, device="cuda")
        x[1] = logits(1, COLS, dt, 52, std=0.01)[0]
        x[2] = (logits(1, COLS, dt, 53).float().round() * 0.5).to(dt)[0]
        x[3, 40000:] = 1.0
        u = [0.0, 0.37, 0.62, 1.0 - 2.0 ** -24]
        run(q, "split flat", x, u)
        run(q, "split flat top-p", x, u, top_p=[0.5, 0.9, 0.25, 0.999])
        run(q, "split flat min-p", x, u, min_p=[1.0, 0.99, 0.05, 0.9], top_p=[1.0, 0.5, 0.99, 0.7])


def test_views_of_wider_rows(q):
    for dt in DTS:
        wide = logits(4, COLS + 9, dt, 54)
        u = [0.1, 0.4, 0.7, 0.95]
        for off in (0, 1, 3, 7):
            run(q, "split view %d" % off, wide[:, off:off + COLS], u, top_p=[0.9, 0.99, 0.2, 1.0])
        run(q, "split view plain", wide[:, 5:5 + COLS], u, min_p=[0.0, 0.0, 0.01, 0.2])
        run(q, "split view greedy", wide[:, 3:3 + COLS], u, temperature=[0.0, 0.5, 0.0, 2.0])


def test_parameters_that_are_not_numbers(q):
    nan = math.nan
    x = logits(5, COLS, torch.float32, 55)
    token, prob = {}, {}
    kw = dict(temperature=dev([nan, 1.0, 1e-30, 1e30, 1.0]), top_p=dev([0.5, nan, 0.9, 0.9, -nan]),
              min_p=dev([0.1, nan, 0.1, 0.0, 2.0]))
    u = dev([0.5, nan, 2.0, -1.0, 0.3])
    for ws in (None, q.sample_workspace(x)):
        token[ws is None], prob[ws is None] = q.quake_sample(x, u, workspace=ws, **kw)
    torch.cuda.synchronize()
    assert torch.equal(token[True], token[False]) and torch.equal(prob[True], prob[False])
    host, got = x.cpu().numpy(), token[True].tolist()
    for r, par in enumerate((dict(temperature=0.0), dict(), dict(temperature=1e-30, top_p=0.9, min_p=0.1),
                             dict(temperature=1e30, top_p=0.9), dict(min_p=1.0))):
        assert got[r] == ref64.sample_row(host[r], [0.5, 0.0, 1.0, 0.0, 0.3][r], mode=2, **par)[0], r


@pytest.mark.parametrize("rows,cols", [(64, 65536), (65, 65536), (32, 65543), (33, 65543), (64, 65535),
                                       (3, 131071)])
def test_both_forms_around_the_switch(q, rows, cols):
    x = logits(rows, cols, torch.bfloat16, rows + cols)
    g = torch.Generator(device="cuda").manual_seed(rows)
    u = torch.rand(rows, generator=g, device="cuda")
    par = dict(top_p=torch.rand(rows, generator=g, device="cuda"),
               min_p=torch.rand(rows, generator=g, device="cuda") * 0.05,
               temperature=torch.rand(rows, generator=g, device="cuda") - 0.1)
    for names in ((), ("top_p",), ("min_p",), ("temperature", "top_p", "min_p")):
        say("switch", rows, cols, names)
        kw = {n: par[n] for n in names}
        a = q.quake_sample(x, u, **kw)
        b = q.quake_sample(x, u, workspace=q.sample_workspace(x), **kw)
        torch.cuda.synchronize()
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("names", [(), ("top_p",), ("min_p",), ("temperature",),
                                   ("temperature", "top_p", "min_p")], ids=str)
def test_graph_streams_and_a_used_workspace(q, names):
    """The split form captured and replayed on changed logits and parameters, its
    workspace full of other calls' words, against one workgroup a row on a stream."""
    rows = 6
    x = logits(rows, COLS, torch.float32, 56)
    ws = q.sample_workspace(x)
    assert ws is not None
    ws.fill_(0xA5)
    u = torch.rand(rows, device="cuda")
    par = {n: torch.full((rows,), 0.9, device="cuda") for n in names}
    token = torch.zeros(rows, dtype=torch.int32, device="cuda")
    prob = torch.zeros(rows, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        q.quake_sample(x, u, token, prob, workspace=ws, **par)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    for i in range(4):
        x.copy_(logits(rows, COLS, torch.float32, 60 + i, std=0.02 if i == 2 else 3.0))
        u.copy_(torch.rand(rows, device="cuda"))
        for n, v in par.items():
            v.copy_(torch.rand(rows, device="cuda") * (0.05 if n == "min_p" else 1.0))
            if n == "temperature":
                v[i::3] = 0.0
        token.fill_(-7)
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = q.quake_sample(x, u, **par)
        with torch.cuda.stream(other):               # eager, with the graph's workspace
            again = q.quake_sample(x, u, workspace=ws, **par)
        side.synchronize()
        other.synchronize()
        assert torch.equal(token, want[0]) and torch.equal(prob, want[1]), i
        assert torch.equal(again[0], want[0]) and torch.equal(again[1], want[1]), i


def _check_exact(row, u, token, top_p, min_p):
    """EXACT's token within what an exponential off by e = 2^-20 of itself allows (the
    hardware's is within 2^-22 of the reference's binary32 value; two such words, and
    sums of them, by less than e). A word is surely kept where no border lies within
    that: before it in the ranking may then come or go 2 e of all mass and the words whose
    weight is within 2 e of its own. The running mass may be off by e of all and by the
    words that are not sure."""
    _, _, upto = ref64.sample_row(row, u, mode=0)
    mass = np.diff(upto, prepend=0).astype(np.float64)
    e, order = 2.0 ** -20, np.argsort(-mass, kind="stable")
    m = mass[order]
    before = np.cumsum(m) - m
    z = m.sum()
    up = -m                                              # ascending
    lo, hi = np.searchsorted(up, -(m * (1 + 2 * e) + 1)), np.searchsorted(up, -(m * (1 - 2 * e) - 1), "right")
    run_m = np.concatenate(([0.0], np.cumsum(m)))
    near = 2 * e * z + (run_m[hi] - run_m[lo]) - m
    goal, least = ref64.fraction(top_p) / 2.0 ** 24 * z, ref64.fraction(min_p) / 2.0 ** 24 * 2.0 ** 40
    sure = (before + near < goal) & (m * (1 - 2 * e) - 1 > least)
    sure[0] = True
    may = (before - near < goal) & (m * (1 + 2 * e) + 1 >= least) & (m > 0)
    unsure = m[may & ~sure].sum()
    kept = np.zeros(len(m))
    kept[order] = np.where(may, m, 0.0)
    upto = np.cumsum(kept)
    slack = 2 * e * z + 2 * unsure
    assert unsure < 1e-3 * z                             # the check means something
    assert kept[token] > 0
    assert upto[token] - kept[token] - slack <= u * upto[-1] <= upto[token] + slack


@pytest.mark.parametrize("cols", [30000, COLS])
def test_exact_mode_filters(q, cols):
    n = 8
    x = logits(n, cols, torch.float32, cols)
    x[6, ::3] = -math.inf
    u = np.random.default_rng(cols).random(n, dtype=np.float32)
    p = [0.9, 0.5, 0.99, 0.2, 1.0, 0.95, 0.8, 1.0]
    m = [0.0, 0.01, 0.001, 0.0, 0.02, 0.05, 0.002, 0.3]
    for tp, mp in ((p, None), (None, m), (p, m)):
        for ws in (None, q.sample_workspace(x)):
            say("exact", cols, tp is not None, mp is not None, ws is not None)
            token, prob = q.quake_sample(x, dev(u.tolist()), top_p=dev(tp), min_p=dev(mp), mode=0, workspace=ws)
            torch.cuda.synchronize()
            for r, tok in enumerate(token.tolist()):
                _check_exact(x[r].cpu().numpy(), float(u[r]), tok, tp[r] if tp else 1.0, mp[r] if mp else 0.0)
        assert ws is None if cols < 65536 else ws is not None


def test_offsets_past_32_bits(q):
    far = (1 << 31) + 24
    buf = torch.empty(2 * far + COLS, dtype=torch.bfloat16, device="cuda")
    x = logits(3, COLS, torch.bfloat16, 57)
    view = buf.as_strided((3, COLS), (far, 1))
    view.copy_(x)
    u = dev([0.2, 0.5, 0.9])
    for par in ({}, dict(top_p=dev([0.9, 0.5, 0.99])), dict(top_k=dev([1, 40, 4000], torch.int32)),
                dict(temperature=dev([0.0, 1.0, 0.0]))):
        for ws in (None, q.sample_workspace(x)):
            say("far rows", list(par), ws is not None)
            want = q.quake_sample(x, u, workspace=ws, **par)
            got = q.quake_sample(view, u, workspace=ws, **par)
            torch.cuda.synchronize()
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
