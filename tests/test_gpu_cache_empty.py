"""Calls of the cache operators that have nothing to do, made as a user's program makes
them: with the workspace that the library asks for, which is none."""
import pytest
import torch

from test_gpu_evict import q  # noqa: F401 (the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("batch,sq", [(0, 1), (0, 0), (2, 0)])
@pytest.mark.parametrize("prefix", [False, True])
def test_empty_steps_with_a_weight(q, batch, sq, prefix):  # noqa: F811
    x = torch.ones((batch, sq, 4, 64), dtype=torch.bfloat16, device="cuda")
    k = torch.ones((batch, 10, 2, 64), dtype=torch.bfloat16, device="cuda")
    pk = torch.ones((1, 6, 2, 64), dtype=torch.bfloat16, device="cuda") if prefix else None
    w = torch.full((batch, 2, 10), 3.0, device="cuda")
    ws = q.attention_shared_workspace(x, k, pk, weigh=True)
    assert ws is None
    o = q.quake_attention_shared(x, k, k.clone(), pk, pk, weight=w, workspace=ws)
    torch.cuda.synchronize()
    assert o.shape == x.shape and (w == 3.0).all()


def test_a_step_with_rows_needs_its_workspace(q):  # noqa: F811
    x, k = (torch.ones((2, n, 2, 64), dtype=torch.bfloat16, device="cuda") for n in (1, 10))
    w = torch.zeros((2, 2, 10), device="cuda")
    with pytest.raises(ValueError, match="a weight needs a workspace"):
        q.quake_attention_shared(x, k, k.clone(), weight=w)
    assert (w == 0).all()
