"""Workspaces of quake_attention_window, quake_sample and quake_distill that share
bytes with an operand are refused (CPU: every call returns before a HIP call)."""
import pytest

from test_abi_decode import A, caller, q, strides, window  # noqa: F401 (q: the fixture)

AT = {n: A + (i + 1 << 22) for i, n in enumerate(("q", "k", "v", "o", "ql", "kl", "x", "u", "token", "prob", "temp",
                                              "p", "m", "idx", "y", "w", "loss", "stats", "grad"))}


def only(names):
    return {n: AT[n] for n in names.split()}


def refused(q, call, need, name, size):
    """The workspace over an operand's first bytes, its last, and all of it."""
    at = AT[name]
    for ws in {at, at - need + 16, (at + size - 1) & ~15, (at + size // 2) & ~15}:
        assert call(ws=ws, nws=need) == q.EINVAL, (name, hex(ws))


@pytest.mark.parametrize("name,size", [("q", 2 * 8 * 64), ("k", 2 * 5000 * 64), ("v", 2 * 5000 * 64),
                                       ("o", 2 * 8 * 64), ("ql", 4), ("kl", 4)])
def test_window(q, name, size):
    call = window(q)
    kw = dict(only("q k v o ql kl"), batch=1, sq=1, skv=5000, heads=8, kv=1, window=5000,
              st=strides(q=(512, 512, 64), o=(512, 512, 64)))
    need = q._size("quake_attention_window_workspace_size", 1, 1, 5000, 8, 1, 64, 5000, 0)
    assert need > 0
    refused(q, lambda **w: call(**dict(kw, sinks=0, **w)), need, name, size)


@pytest.mark.parametrize("name,size", [("x", 4 * (100000 + 90000)), ("u", 8), ("token", 8), ("prob", 8),
                                       ("temp", 8), ("p", 8), ("m", 8)])
def test_sample(q, name, size):
    call = caller(q.lib.quake_sample,
                  dict(only("x u token prob temp p m"), rows=2, cols=90000, ldx=100000, k=None, dt=0, mode=2,
                       stream=None), "x u token prob rows cols ldx temp k p m dt mode ws nws stream")
    need = q._size("quake_sample_workspace_size", 2, 90000)
    assert need > 0
    refused(q, call, need, name, size)


@pytest.mark.parametrize("name,size", [("x", 2 * (100000 + 90000)), ("grad", 2 * (110000 + 90000)),
                                       ("idx", 4 * (30 + 20)), ("y", 4 * (25 + 20)), ("w", 8), ("loss", 8),
                                       ("stats", 16)])
def test_distill(q, name, size):
    call = caller(q.lib.quake_distill,
                  dict(only("x idx y w loss stats grad"), rows=2, cols=90000, k=20, ldx=100000, ldi=30, ldy=25,
                       ldg=110000, dt=2, ydt=0, mode=2, t=1.0, stream=None),
                  "x idx y w loss stats grad rows cols k ldx ldi ldy ldg dt ydt mode t ws nws stream")
    need = q._size("quake_distill_workspace_size", 2, 90000)
    assert need > 0
    refused(q, call, need, name, size)
