"""quake_sample on the GPU against its definition in whole numbers: the same token
(the bit constructions' weights are reproducible) and the same probability."""
import math

import numpy as np
import pytest
import torch

import ref64
from gpu_util import say

pytestmark = pytest.mark.gpu
DTS = [torch.float32, torch.bfloat16, torch.float16]


@pytest.fixture(scope="module")
def q():
    from paper_2412_00408_amd import quake
    return quake


def logits(rows, cols, dt, seed, std=3.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn((rows, cols), generator=g, device="cuda").mul_(std).to(dt)


def dev(v, dt=torch.float32):
    return None if v is None else torch.tensor(v, dtype=dt, device="cuda")


def run(q, name, x, u, temperature=None, top_k=None, top_p=None, min_p=None, mode=2):
    """Every row against ref64.sample_row, with a workspace and without."""
    say(name, tuple(x.shape), x.dtype, "mode", mode)
    rows = x.shape[0]
    for ws in (None, q.sample_workspace(x)):
        token, prob = q.quake_sample(x, dev(u), temperature=dev(temperature),
                                     top_k=dev(top_k, torch.int32), top_p=dev(top_p),
                                     min_p=dev(min_p), mode=mode, workspace=ws)
        torch.cuda.synchronize()
        token, prob, host = token.tolist(), prob.tolist(), x.float().cpu().numpy()
        for r in range(rows):
            par = dict(temperature=1.0 if temperature is None else temperature[r],
                       top_k=0 if top_k is None else top_k[r],
                       top_p=1.0 if top_p is None else top_p[r],
                       min_p=0.0 if min_p is None else min_p[r])
            want, p, _ = ref64.sample_row(host[r], u[r], mode=mode, **par)
            assert token[r] == want, (name, r, token[r], want, par, u[r], ws is not None)
            assert abs(prob[r] - p) <= 2.0 ** -23 * p, (name, r, prob[r], p)


@pytest.mark.parametrize("dt", DTS, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("cols", [1, 2, 63, 64, 65, 1000, 1023, 4097, 32001, 50257, 128256])
def test_filters(q, cols, dt):
    rng = np.random.default_rng(cols)
    x = logits(12, cols, dt, cols)
    u = rng.random(12, dtype=np.float32).tolist()
    u[0], u[1] = 0.0, 1.0 - 2.0 ** -24
    k = [1, 2, 3, 5, 50, 100, 400, cols, cols - 1, 0, -3, 1500]
    p = [0.9, 0.5, 0.99, 1.0, 0.0, -1.0, 0.3, 0.95, 0.999, 0.1, 2.0, 0.7]
    m = [0.0, 0.1, 0.05, 1.0, 2.0, -1.0, 0.001, 0.3, 1e-6, 0.01, 0.5, 0.02]
    temp = [1.0, 0.7, 1.3, 0.0, 0.1, 2.0, 0.5, -1.0, 1.0, 0.9, 4.0, 0.01]
    mode = 1 + cols % 3
    run(q, "none", x, u, mode=mode)
    run(q, "temperature", x, u, temperature=temp, mode=mode)
    run(q, "top-k", x, u, top_k=k, mode=mode)
    run(q, "top-p", x, u, top_p=p, mode=mode)
    run(q, "min-p", x, u, min_p=m, mode=mode)
    run(q, "all", x, u, temperature=temp, top_k=k, top_p=p, min_p=m, mode=mode)


@pytest.mark.parametrize("mode", [1, 2, 3])
def test_ties_go_to_the_lowest_index(q, mode):
    # few distinct values, so every border falls among equal weights
    x = (logits(8, 5000, torch.float32, 11).round() * 0.5).contiguous()
    u = np.linspace(0.01, 0.99, 8, dtype=np.float32).tolist()
    run(q, "ties k", x, u, top_k=[1, 2, 7, 50, 333, 1000, 2500, 4999], mode=mode)
    run(q, "ties p", x, u, top_p=[0.01, 0.1, 0.2, 0.4, 0.6, 0.8, 0.9, 0.999], mode=mode)
    run(q, "ties kp", x, u, top_k=[100] * 8, top_p=[0.01, 0.1, 0.2, 0.4, 0.6, 0.8, 0.9, 0.999], mode=mode)
    flat = torch.full((4, 70000), 1.25, dtype=torch.bfloat16, device="cuda")
    run(q, "flat", flat, [0.0, 0.3, 0.5, 0.999], top_k=[1, 600, 0, 69999], top_p=[0.5, 0.9, 0.25, 0.75],
        mode=mode)


def test_wide_nucleus(q):
    # almost flat rows: the kept words are tens of thousands
    x = logits(4, 100003, torch.float32, 12, std=0.05)
    run(q, "wide", x, [0.1, 0.5, 0.7, 0.99], top_p=[0.9, 0.5, 0.99, 0.1], top_k=[0, 90000, 3000, 0])


def test_longest_rows(q):
    x = logits(2, 1 << 22, torch.bfloat16, 21)
    u = [0.3, 0.8]
    run(q, "longest", x, u)
    run(q, "longest top-p", x, u, top_p=[0.9, 0.2], min_p=[0.0, 0.001])
    run(q, "longest top-k", x, u, top_k=[60, 1], temperature=[0.7, 0.0])
    run(q, "longest greedy", x, u, temperature=[0.0, 1.0])


def test_split_rows_with_greedy_rows_among_them(q):
    for dt in DTS:
        x = logits(6, 70001, dt, 22)
        x[1, 60000:60010] = x[1].max() + 1           # equal largest words
        x[1, 30:33] = x[1, 60000]
        x[2] = -math.inf
        x[3, 5] = math.inf
        u = [0.1, 0.9, 0.5, 0.5, 0.7, 0.2]
        temp = [0.0, 0.0, 0.0, 0.0, 1.0, -3.0]
        run(q, "greedy among", x, u, temperature=temp)
        run(q, "greedy among, top-p", x, u, temperature=temp, top_p=[0.9] * 6, min_p=[0.02] * 6)


def test_masked_words_infinities_and_nan(q):
    inf, nan = math.inf, math.nan
    for cols in (40, 20000, 40000):
        x = logits(7, cols, torch.float32, 13)
        x[0] = -inf                                  # nothing allowed
        x[1, 1:] = -inf                              # one word
        x[1, 0] = -3e38                              # far below the rest of the batch
        x[2, ::2] = -inf
        x[3, 5] = nan
        x[3, 7:30] = nan
        x[4, 9] = inf                                # certain
        x[4, 21] = inf
        x[5] = torch.finfo(torch.float32).min        # the type's lowest value everywhere
        x[6, :] = nan
        u = [0.5] * 7
        run(q, "masked", x, u)
        run(q, "masked filters", x, u, top_k=[3] * 7, top_p=[0.8] * 7, min_p=[0.01] * 7)
        run(q, "masked greedy", x, u, temperature=[0.0] * 7)


def test_parameters_that_are_not_numbers(q):
    x = logits(6, 3000, torch.float32, 14)
    nan, inf = math.nan, math.inf
    host = x.cpu().numpy()
    cases = [dict(temperature=nan), dict(temperature=inf), dict(top_p=nan), dict(min_p=nan),
             dict(temperature=1e-30), dict(temperature=1e30)]
    cols = {k: [c.get(k, d) for c in cases] for k, d in
            (("temperature", 1.0), ("top_p", 1.0), ("min_p", 0.0))}
    token, _ = q.quake_sample(x, dev([0.5, 0.5, nan, 2.0, -1.0, inf]),
                              **{k: dev(v) for k, v in cols.items()})
    got = token.tolist()
    uu = [0.5, 0.5, 0.0, 1.0, 0.0, 1.0]
    for r in range(6):
        par = {k: v[r] for k, v in cols.items()}
        if math.isnan(par["top_p"]):
            par["top_p"] = 1.0
        if math.isinf(par["temperature"]):
            par["temperature"] = 1e38
        assert got[r] == ref64.sample_row(host[r], uu[r], mode=2, **par)[0], (r, par)


def test_exact_mode(q):
    # w is the hardware exponential: at most 2^-22 from the reference's, so the
    # running sum may differ by 2^-21 of it at any word
    x = logits(16, 30000, torch.float32, 15)
    u = np.random.default_rng(3).random(16, dtype=np.float32).tolist()
    for k in (0, 20):
        token, _ = q.quake_sample(x, dev(u), top_k=dev([k] * 16, torch.int32), mode=0)
        for r, tok in enumerate(token.tolist()):
            _, _, upto = ref64.sample_row(x[r].cpu().numpy(), u[r], top_k=k, mode=0)
            goal, slack = u[r] * float(upto[-1]), 2.0 ** -20 * float(upto[-1])
            before = float(upto[tok - 1]) if tok else 0.0
            assert before - slack <= goal <= float(upto[tok]) + slack, (r, k)


def test_strided_and_unaligned_rows(q):
    wide = logits(9, 1000 + 7, torch.bfloat16, 16)
    u = np.linspace(0.05, 0.95, 9, dtype=np.float32).tolist()
    for off in (0, 1, 3):
        run(q, "view", wide[:, off:off + 1000], u, top_k=[40] * 9, top_p=[0.9] * 9)
    big = logits(5, 40000 + 9, torch.float32, 17)
    run(q, "long view", big[:, 3:40003], u[:5], top_k=[40] * 5, top_p=[0.9] * 5)
    run(q, "long view", big[:, 3:40003], u[:5], top_p=[0.9] * 5)


def test_many_rows(q):
    x = logits(3000, 300, torch.bfloat16, 18)
    u = np.random.default_rng(4).random(3000, dtype=np.float32).tolist()
    run(q, "rows", x, u, top_k=[20] * 3000, top_p=[0.9] * 3000)
    x = logits(1500, 20000, torch.bfloat16, 19)
    u = torch.rand(1500, device="cuda")
    ws = q.sample_workspace(x)
    k = torch.full((1500,), 40, dtype=torch.int32, device="cuda")
    a = q.quake_sample(x, u, top_k=k)
    b = q.quake_sample(x, u, top_k=k, workspace=ws)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_distribution(q):
    # 2^16 draws of one row: every word as often as its probability, within six
    # standard deviations
    n = 1 << 16
    row = torch.tensor([2.0, 1.0, 0.0, -1.0, 1.5, -math.inf], device="cuda")
    u = (torch.arange(n, device="cuda").float() + 0.5) / n
    token, _ = q.quake_sample(row.expand(n, 6).contiguous(), u)
    count = torch.bincount(token.long(), minlength=6).double() / n
    w = ref64.real_exp2((row.double() - 2.0) / ref64.LN2, 2)
    assert ((count - w / w.sum()).abs() < 2.0 / n + 1e-5).all() and count[5] == 0


def test_graph_and_streams(q):
    for cols in (5000, 60000):
        x = logits(6, cols, torch.float32, 20)
        ws = q.sample_workspace(x)
        u = torch.rand(6, device="cuda")
        k = torch.full((6,), 30, dtype=torch.int32, device="cuda")
        p = torch.full((6,), 0.9, device="cuda")
        token = torch.zeros(6, dtype=torch.int32, device="cuda")
        prob = torch.zeros(6, device="cuda")
        kw = dict(top_k=k, top_p=p, workspace=ws)
        q.quake_sample(x, u, token, prob, **kw)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            q.quake_sample(x, u, token, prob, **kw)
        side = torch.cuda.Stream()
        for i in range(4):
            x.copy_(logits(6, cols, torch.float32, 30 + i))
            u.copy_(torch.rand(6, device="cuda"))
            k.fill_(0 if i == 2 else 20 * i + 1)
            graph.replay()
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                want = q.quake_sample(x, u, **kw)
            side.synchronize()
            assert torch.equal(token, want[0]) and torch.equal(prob, want[1])
