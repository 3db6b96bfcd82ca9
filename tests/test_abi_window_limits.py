"""quake_attention_window's limits on the CPU: the largest grid, outputs whose rows
overlap, workspaces that overlap an operand. Every call below returns before a HIP
call or a launch."""
import pytest

from test_abi_decode import q, strides, window  # noqa: F401 (q: the fixture)

SOUND = dict(q=(1024, 256, 64), o=(1024, 256, 64), k=(12800, 128, 64), v=(12800, 128, 64))


def sound(**kw):
    return strides(**dict(SOUND, **kw))


# batch, sq, heads, kv_heads of 2^24 tiles of 32 rows: 2^32 threads, one more than a
# launch takes
@pytest.mark.parametrize("b,sq,h,hk", [(1 << 24, 1, 1, 1), (1 << 20, 1, 16, 16), (1, 1 << 24, 32, 32),
                                       (1 << 23, 33, 1, 1), (1 << 24, 1, 32, 1)], ids=str)
def test_the_largest_grid(q, b, sq, h, hk):
    size = "quake_attention_window_workspace_size"
    with pytest.raises(q.QuakeError):
        q._size(size, b, sq, 10, h, hk, 64, 10, 0)
    st = sound(q=(h * sq * 64, h * 64, 64), o=(h * sq * 64, h * 64, 64))
    assert window(q)(batch=b, sq=sq, heads=h, kv=hk, skv=10, st=st) == q.EINVAL
    one_less = (b - 1, sq) if b > 1 else (b, sq - 32)
    assert q._size(size, *one_less, 10, h, hk, 64, 10, 0) == 0
