"""Where quake_attention_window writes: outputs in any order of batch, tokens and heads,
as slices of wider buffers, beside what they leave alone."""
import pytest
import torch

from test_gpu_window import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def q():
    from paper_2412_00408_amd import quake
    return quake


@pytest.mark.parametrize("order", [(0, 1, 2), (0, 2, 1), (1, 0, 2), (1, 2, 0), (2, 0, 1), (2, 1, 0)], ids=str)
@pytest.mark.parametrize("sq", [1, 5, 140])
def test_orders_and_slices(q, order, sq):
    b, skv, h, hk, d = 3, 200, 4, 2, 64
    x = make(b, sq, skv, h, hk, d, torch.bfloat16, 31)
    want = q.quake_attention_window(*x, window=100, sinks=3)
    sizes = (b, sq, h)
    back = [order.index(i) for i in range(3)]
    for extra, step in ((0, 1), (1, 1), (0, 2)):        # packed, padded, every other one
        buf = torch.full([(sizes[i] + extra) * step for i in order] + [d + 8 * extra], 7.0,
                         dtype=torch.bfloat16, device="cuda")
        o = buf.permute(*back, 3)[:b * step:step, :sq * step:step, :h * step:step, :d]
        q.quake_attention_window(*x, o, window=100, sinks=3)
        assert torch.equal(o, want)
        o.fill_(7.0)
        assert (buf == 7.0).all()
