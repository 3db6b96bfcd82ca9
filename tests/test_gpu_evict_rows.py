"""quake_cache_evict on rows on both sides of the lengths at which the choice holds its slots
in other ways: 256 threads with 16 slots each (4096), 1024 with 16 (16384) and with 40
(40960), longer rows read again. Bit for bit against the choice by whole numbers, and a
row that ragged batches mix."""
import pytest
import torch

from test_gpu_evict import both, cache, q  # noqa: F401 (q: the fixture)

pytestmark = pytest.mark.gpu

LIMITS = [4095, 4096, 4097, 16383, 16384, 16385, 22013, 40959, 40960, 40961]


@pytest.mark.parametrize("n", LIMITS)
@pytest.mark.parametrize("kind", ["spread", "ties", "one", "odd"])
def test_rows_about_the_limits(q, n, kind):  # noqa: F811
    for budget, sinks, recent in ((n // 3, 4, 100), (n - 1, 0, 0), (1, 0, 0), (n // 2, n // 4, n // 2 - n // 4)):
        both(q, "%d %s budget %d" % (n, kind, budget), *cache(1, n, 2, 8, torch.bfloat16, n, kind), budget, sinks,
             recent, None)


@pytest.mark.parametrize("kind", ["spread", "ties", "one"])
@pytest.mark.parametrize("slots", [41000, 40960, 16400, 4100])
def test_ragged_batches_about_the_limits(q, slots, kind):  # noqa: F811
    lens = [n for n in LIMITS if n <= slots] + [slots, slots + 7, 4000, 1000, 999, 1, 0, -1]
    lens = torch.tensor(lens, dtype=torch.int32, device="cuda")
    both(q, "%d slots %s" % (slots, kind), *cache(lens.numel(), slots, 1, 64, torch.float16, 5, kind), 1000, 3, 20, lens)
