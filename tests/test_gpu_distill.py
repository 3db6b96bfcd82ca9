"""quake_distill and quake_distill_grad on the GPU against the formulas in 64 bits
and against differences of the loss, within the bounds ref64.distill derives."""
import math

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


def make(rows, cols, k, dt, seed=0, ydt=torch.float32):
    g = torch.Generator(device="cuda").manual_seed(seed + rows * 131 + cols)
    x = torch.randn((rows, cols), generator=g, device="cuda").mul_(3.0)
    idx = torch.randint(cols, (rows, k), generator=g, device="cuda", dtype=torch.int32)
    y = torch.randn((rows, k), generator=g, device="cuda").mul_(2.0).add_(5.0).to(ydt)
    w = torch.rand(rows, generator=g, device="cuda") + 0.5
    return x.to(dt), idx, y, w


def near(name, got, want, bound):
    off = (got.double() - want).abs()
    bad = ~((off <= bound) | (got.double() == want))
    if bad.any():
        at = tuple(bad.nonzero()[0].tolist())
        raise AssertionError("%s: %d of %d out of bound, first at %s: %s for %s, bound %s" % (
            name, int(bad.sum()), bad.numel(), at, got[at].item(), want[at].item(), bound[at].item()))


def run(q, name, x, idx, y, w, mode, t):
    say(name, tuple(x.shape), tuple(idx.shape), x.dtype, "mode", mode)
    loss, grad, lb, gb = ref64.distill(x, idx, y, mode, t, w)
    for ws in (None, q.distill_workspace(x)):
        got, stats, g = q.quake_distill(x, idx, y, weight=w, grad=True, mode=mode, t=t, workspace=ws)
        torch.cuda.synchronize()
        near(name + " loss", got, loss, lb)
        near(name + " grad", g, grad, gb)
        only, stats2, none = q.quake_distill(x, idx, y, mode=mode, t=t, workspace=ws)
        assert none is None and torch.equal(only, got) and torch.equal(stats, stats2)
        later = q.quake_distill_grad(x, idx, y, stats, weight=w, mode=mode, t=t)
        assert torch.equal(later, g)


@pytest.mark.parametrize("dt", DTS, ids=["f32", "bf16", "f16"])
@pytest.mark.parametrize("rows,cols,k", [
    (1, 1, 1), (3, 2, 2), (5, 7, 3), (4, 64, 1), (3, 1000, 20), (2, 4099, 64), (7, 8191, 5),
    (2, 16384, 1024), (3, 32001, 100), (2, 50257, 513), (1, 128256, 64), (600, 515, 33)])
def test_shapes(q, rows, cols, k, dt):
    for mode in (0, 1, 2, 3):
        run(q, "distill", *make(rows, cols, k, dt), mode, 0.5 if mode & 1 else 1.0)


@pytest.mark.parametrize("ydt", DTS, ids=["f32", "bf16", "f16"])
def test_teacher_formats_and_strides(q, ydt):
    x, idx, y, w = make(6, 3000, 40, torch.bfloat16, 1, ydt)
    run(q, "teacher format", x, idx[:, :17], y[:, 3:20], w, 2, 0.7)     # rows of wider matrices
    wide = torch.randn(6, 3011, device="cuda").to(torch.bfloat16)
    for off in (0, 1, 5):
        run(q, "offset rows", wide[:, off:off + 3000], idx, y, w, 2, 0.7)


def test_padding_repeated_words_and_empty_rows(q):
    for dt in DTS:
        x, idx, y, w = make(8, 3001, 24, dt, 2)
        idx[0] = -1                                   # no entry
        idx[1, 5:] = -1
        idx[2, ::3] = 3001                            # outside the vocabulary
        idx[3] = 77                                   # one word 24 times
        idx[4, 12:] = idx[4, :12]                     # every word twice
        y[5] = -math.inf                              # entries without mass
        y[6, 1:] = -math.inf
        w[7] = 0.0
        run(q, "padded", x, idx, y, w, 2, 1.0)
        loss, _, grad = q.quake_distill(x, idx, y, weight=w, grad=True)
        for r in (0, 5):
            assert loss[r] == 0 and (grad[r] == 0).all()
        assert (grad[7] == 0).all() and loss[7] != 0
        empty = torch.empty((8, 0), dtype=torch.int32, device="cuda")
        loss, _, grad = q.quake_distill(x, empty, empty.float(), grad=True)
        assert (loss == 0).all() and (grad == 0).all()


def test_masked_logits(q):
    for cols in (300, 30000):
        x, idx, y, w = make(5, cols, 10, torch.float32, 3)
        x[0, ::2] = -math.inf
        idx[0] = idx[0] | 1                           # entries at words that are allowed
        x[1, int(idx[1, 0])] = -math.inf              # one that is not
        x[2] = -math.inf
        x[3] = torch.finfo(torch.float32).min / 1e33  # far, but within the range
        ws = q.distill_workspace(x)
        loss, _, grad = q.quake_distill(x, idx, y, weight=w, grad=True, workspace=ws)
        want, wgrad, lb, gb = ref64.distill(x[:1], idx[:1], y[:1], 2, 1.0, w[:1])
        near("allowed loss", loss[:1], want, lb)
        near("allowed grad", grad[:1], wgrad, gb)
        assert loss[1] == math.inf and loss[2] == math.inf
        assert torch.isfinite(grad[:4]).all()
        rest = ref64.distill(x[4:], idx[4:], y[4:], 2, 1.0, w[4:])
        near("beside them", grad[4:], rest[1], rest[3])


def test_in_place_and_same_bits(q):
    for rows, cols in ((3, 40001), (600, 333)):
        for dt in DTS:
            x, idx, y, w = make(rows, cols, 50, dt, 4)
            ws = q.distill_workspace(x)
            want = q.quake_distill(x, idx, y, weight=w, grad=True, workspace=ws)
            for _ in range(2):
                c = x.clone()
                loss, _, g = q.quake_distill(c, idx, y, weight=w, grad=c, workspace=ws)
                assert g is c and torch.equal(g, want[2]) and torch.equal(loss, want[0])
            c = x.clone()
            q.quake_distill_grad(c, idx, y, want[1], weight=w, grad=c)
            assert torch.equal(c, want[2])
            out = torch.full((rows, cols + 9), 5.0, dtype=dt, device="cuda")
            q.quake_distill(x, idx, y, weight=w, grad=out[:, 4:cols + 4], workspace=ws)
            assert torch.equal(out[:, 4:cols + 4], want[2])
            assert (out[:, :4] == 5).all() and (out[:, cols + 4:] == 5).all()


@pytest.mark.parametrize("mode", [0, 1, 2])
def test_gradient_against_differences(q, mode):
    """Central differences of the kernel's loss. The exact mode's gradient is the
    loss's: off by h^2/6 of the third derivative (at most t^3 / 4 for a softmax) and by
    the loss's error over h. The other modes' formula keeps the exponential's own
    error out of the derivative: d/dx log S = t Q'/S where the formula has t Q/S, and
    Q' lies within 1/(1+f) ln2^-1 .. of Q, at most 44.3 % (first order), 6.2 %
    (refined: 2 a^2 / ((a^2 + 2) ln 2) at a = 2 over 1.5 ...) of q."""
    rows, cols, k, h = 4, 30, 6, 2.0 ** -4
    x, idx, y, _ = make(rows, cols, k, torch.float32, 5)
    x = (x * 0.5).contiguous()
    _, _, g = q.quake_distill(x, idx, y, grad=True, mode=mode)
    a = torch.arange(cols, device="cuda")
    plus = x[:, None, :].repeat(1, cols, 1)
    minus = plus.clone()
    plus[:, a, a] += h
    minus[:, a, a] -= h
    rep = [v.repeat_interleave(cols, 0) for v in (idx, y)]
    lp = q.quake_distill(plus.view(-1, cols), *rep, mode=mode)[0].double()
    lm = q.quake_distill(minus.view(-1, cols), *rep, mode=mode)[0].double()
    diff = ((lp - lm) / (2 * h)).view(rows, cols)
    loss, grad, lb, gb = ref64.distill(x, idx, y, mode, 1.0)
    soft = ref64.real_exp2(x.double() / ref64.LN2, mode)
    soft = soft / soft.sum(1, keepdim=True)
    # Q'/Q - 1 over a binade: first order 1/(ln2 (1+f)) - 1 in [-0.279, 0.443]; refined
    # 2a/(ln2 (a^2+2)) - 1, largest at a = 1 and 2: -0.0383, at sqrt2: 0.0202
    share = {0: 0.0, 1: 0.443, 2: 0.0383}[mode]
    slack = share * soft * 1.1 + h * h / 24 + gb + (lb.max() if mode == 0 else 2 * ref64.ARG * 4) / h
    assert ((diff - g.double()).abs() <= slack).all()


def test_offsets_past_32_bits(q):
    rows, cols, k = 3, 5000, 20
    far = (1 << 31) + 8
    buf = torch.empty(2 * far + cols, dtype=torch.bfloat16, device="cuda")
    x, idx, y, w = make(rows, cols, k, torch.bfloat16, 6)
    want = q.quake_distill(x, idx, y, weight=w, grad=True)
    view = buf.as_strided((rows, cols), (far, 1))
    view.copy_(x)
    loss, _, g = q.quake_distill(view, idx, y, weight=w, grad=view)
    assert torch.equal(loss, want[0]) and torch.equal(g, want[2])


def test_graph(q):
    for rows, cols in ((4, 40000), (520, 700)):
        x, idx, y, w = make(rows, cols, 30, torch.bfloat16, 7)
        ws = q.distill_workspace(x)
        g = torch.zeros_like(x)
        q.quake_distill(x, idx, y, weight=w, grad=g, workspace=ws)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            loss, stats, _ = q.quake_distill(x, idx, y, weight=w, grad=g, workspace=ws)
        for i in range(4):
            n = make(rows, cols, 30, torch.bfloat16, 40 + i)
            for a, c in zip((x, idx, y, w), n):
                a.copy_(c)
            g.fill_(9.0)
            graph.replay()
            torch.cuda.synchronize()
            want = q.quake_distill(x, idx, y, weight=w, grad=True, workspace=ws)
            assert torch.equal(loss, want[0]) and torch.equal(g, want[2])
