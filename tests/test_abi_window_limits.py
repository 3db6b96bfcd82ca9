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


@pytest.mark.parametrize("o", [
    (1024, 64, 64),        # tokens as far apart as heads: heads fall on the next tokens
    (1024, 128, 64), (1024, 192, 64), (1024, 64, 256 - 8), (256, 256, 64), (1000, 256, 64),
    (64, 1024, 64), (1024, 248, 64), (0, 256, 64), (1760, 64, 504)], ids=str)
def test_outputs_whose_rows_overlap(q, o):
    # batch 2, sq 4, heads 4, dim 64
    assert window(q)(st=sound(o=o)) == q.EINVAL


@pytest.mark.parametrize("bad", [
    dict(batch=-1), dict(sq=-1), dict(skv=-1), dict(heads=0), dict(kv=0), dict(kv=3), dict(dim=32),
    dict(window=0), dict(window=1 << 31), dict(sinks=-1), dict(sinks=1 << 31), dict(t=0.0), dict(t=3e38),
    dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=65544), dict(k=65538), dict(v=65540),
    dict(o=65544), dict(ql=65538), dict(kl=65537), dict(ws=65540), dict(nws=-1),
    dict(st=dict(q=(64, 60, 64))), dict(st=dict(k=(64, -64, 64))), dict(st=dict(k=(64, (1 << 24) + 8, 64))),
    dict(st=dict(v=(64, (1 << 24) + 8, 64))), dict(st=dict(v=(4, 64, 64))), dict(st=dict(o=(-1024, 256, 64))),
    dict(st=dict(o=(1024, 256, 65))), dict(st=dict(o=(1024, 256, 0))), dict(st=dict(q=(1 << 62, 64, 64)))],
    ids=str)
def test_each_refusal_beside_sound_strides(q, bad):
    kw = dict(bad, st=sound(**bad.get("st", {})))
    assert window(q)(**kw) == q.EINVAL
