"""What the training operators refuse, on the host before anything is launched
(no GPU needed: the addresses are never read)."""
import ctypes

import numpy as np
import pytest

from paper_2607_28940_amd import transx as T

A = 0x7F0000000000  # a device address that no call here reaches


@pytest.fixture(scope="module")
def L():
    return T.lib()


def _cfg(dtype=T.TX_BF16, H=4, G=2, dh=64, R=16, scale=0.0):
    return T.AttnConfig(dtype, H, G, dh, R, scale)


def _rows(H=4, dh=64, data=A, row=None, head=None):
    return T.Rows(data, H * dh if row is None else row, dh if head is None else head)


def _rel(L, backward=False, cfg=None, off=(0, 5, 9), n=None, ws=A, ws_bytes=1 << 40, rel=A, drel=A, lse=A, lse_stride=9,
         q=None, k=None, v=None, out=None, dq=None, dk=None, dv=None):
    cfg = cfg or _cfg()
    off = T._i64(off)
    x = dict(q=q or _rows(), k=k or _rows(2), v=v or _rows(2), out=out or _rows())
    g = dict(do=_rows(), dq=dq or _rows(), dk=dk or _rows(2), dv=dv or _rows(2))
    B = ctypes.byref
    args = [B(cfg), len(off) - 1 if n is None else n, T._p(off, T.I64P), B(x["q"]), B(x["k"]), B(x["v"]), T.VP(rel),
            B(x["out"]), T.VP(lse), lse_stride]
    if backward:
        args += [B(v) for v in g.values()] + [T.VP(drel)]
        return L.tx_rel_attn_backward(*args, T.VP(ws), ws_bytes, None)
    return L.tx_rel_attn_forward(*args, T.VP(ws), ws_bytes, None)


def _event(L, backward=False, cfg=None, ko=(0, 5, 9), eo=(0, 1, 3), qo=(0, 2, 4, 7), pre=(5, 1, 0), ws=A,
           ws_bytes=1 << 40, lse_stride=7):
    cfg = cfg or _cfg(R=0)
    a = [T._i64(x) for x in (ko, eo, qo, pre)]
    B = ctypes.byref
    t = [B(_rows()), B(_rows(2)), B(_rows(2)), B(_rows())]
    args = [B(cfg), len(ko) - 1, *[T._p(x, T.I64P) for x in a], *t, T.VP(A), lse_stride]
    if backward:
        args += [B(_rows()), B(_rows()), B(_rows(2)), B(_rows(2))]
        return L.tx_event_attn_backward(*args, T.VP(ws), ws_bytes, None)
    return L.tx_event_attn_forward(*args, T.VP(ws), ws_bytes, None)


@pytest.mark.parametrize("backward", [False, True])
def test_attention_config(L, backward):
    I, U = T.TX_E_INVALID, T.TX_E_UNSUPPORTED
    for cfg, code in ((_cfg(dtype=7), I), (_cfg(H=0), I), (_cfg(H=3, G=2), I), (_cfg(G=0), I), (_cfg(dh=48), U),
                      (_cfg(dh=256), U), (_cfg(R=-1), I), (_cfg(R=2049), U), (_cfg(scale=-1.0), I),
                      (_cfg(scale=float("nan")), I), (_cfg(scale=float("inf")), I)):
        assert _rel(L, backward, cfg=cfg) == code, L.tx_last_error()
        off = T._i64([0, 4])
        assert L.tx_rel_attn_workspace_bytes(ctypes.byref(cfg), int(backward), 1, T._p(off, T.I64P)) == 0
    assert _event(L, backward, cfg=_cfg(R=1)) == I
    assert L.tx_rel_attn_forward(None, 0, None, None, None, None, None, None, None, 0, None, 0, None) == I


@pytest.mark.parametrize("backward", [False, True])
def test_attention_offsets(L, backward):
    I, U = T.TX_E_INVALID, T.TX_E_UNSUPPORTED
    for off, code in (((0, 5, 4), I), ((-1, 5, 9), I), ((0, 5, 1 << 31), U)):
        assert _rel(L, backward, off=off, lse_stride=1 << 40) == code, off
    assert _rel(L, backward, n=-1) == I
    assert _rel(L, backward, lse_stride=8) == I
    for kw in (dict(ko=(0, 5, 4)), dict(eo=(0, 2, 1)), dict(eo=(1, 1, 3)), dict(qo=(0, 2, 1, 7)), dict(pre=(6, 1, 0)),
               dict(pre=(5, -1, 0)), dict(pre=(5, 1, 5)), dict(lse_stride=6)):
        assert _event(L, backward, **kw) == I, kw


@pytest.mark.parametrize("backward", [False, True])
def test_attention_tensors(L, backward):
    I, U = T.TX_E_INVALID, T.TX_E_UNSUPPORTED
    bad = dict(null=_rows(data=None), misaligned=_rows(data=A + 8), row=_rows(row=260), head=_rows(head=68),
               negative=_rows(row=-256), huge=_rows(row=(16 << 20)))
    for name, t in bad.items():
        want = U if name == "huge" else I
        for arg in ("q", "k", "v", "out") + (("dq", "dk", "dv") if backward else ()):
            assert _rel(L, backward, **{arg: t}) == want, (name, arg, L.tx_last_error())
    # overlapping rows or heads may be read, not written
    for t in (_rows(row=0), _rows(row=64), _rows(head=0), _rows(head=32)):
        for arg in ("dq", "dk", "dv") if backward else ("out",):
            assert _rel(L, backward, **{arg: t}) == I, arg
            assert b"overlap" in L.tx_last_error()
    assert _rel(L, backward, rel=None) == I and _rel(L, backward, lse=None) == I
    if backward:
        assert _rel(L, backward, drel=None) == I


@pytest.mark.parametrize("backward", [False, True])
def test_attention_workspace(L, backward):
    off = T._i64([0, 5, 9])
    c = _cfg()
    need = L.tx_rel_attn_workspace_bytes(ctypes.byref(c), int(backward), 2, T._p(off, T.I64P))
    assert need > 0
    assert _rel(L, backward, ws=None) == T.TX_E_INVALID
    assert _rel(L, backward, ws=A + 16) == T.TX_E_INVALID
    assert _rel(L, backward, ws_bytes=need - 1) == T.TX_E_NOMEM
    assert _event(L, backward, ws_bytes=16) == T.TX_E_NOMEM


def _pref(L, backward=False, dtype=T.TX_F32, k=4, beta=0.1, eps=0.0, off=(0, 2, 5), ld=4, ldd=4, logits=A, act=A,
          ws=A, ws_bytes=1 << 40, f32=A, dlogits=A):
    c = T.PreferenceConfig(dtype, k, beta, eps)
    off = T._i64(off)
    P, op = len(off) // 2, T._p(off, T.I64P)
    if backward:
        return L.tx_preference_backward(ctypes.byref(c), P, op, T.VP(logits), ld, T.VP(act), None, T.VP(f32), T.VP(A),
                                        T.VP(A), T.VP(dlogits), ldd, T.VP(ws), ws_bytes, None)
    return L.tx_preference_forward(ctypes.byref(c), P, op, T.VP(logits), ld, T.VP(act), None, T.VP(f32), T.VP(A),
                                   T.VP(A), T.VP(ws), ws_bytes, None)


@pytest.mark.parametrize("backward", [False, True])
def test_preference(L, backward):
    I = T.TX_E_INVALID
    for kw in (dict(dtype=5), dict(k=0), dict(beta=float("nan")), dict(beta=float("inf")), dict(eps=-0.1),
               dict(eps=1.1), dict(eps=float("nan")), dict(off=(0, 5, 2)), dict(off=(-1, 2, 5)), dict(ld=3),
               dict(logits=None), dict(logits=A + 2), dict(act=None), dict(act=A + 1), dict(f32=None),
               dict(f32=A + 2), dict(ws=None), dict(ws=A + 8)):
        assert _pref(L, backward, **kw) == I, (kw, L.tx_last_error())
    assert _pref(L, backward, off=(0, 2, 1 << 31)) == T.TX_E_UNSUPPORTED
    assert _pref(L, backward, ws_bytes=64) == T.TX_E_NOMEM
    if backward:
        for kw in (dict(ldd=3), dict(dlogits=None), dict(dlogits=A + 1)):
            assert _pref(L, True, **kw) == I, kw


def test_python_arguments():
    """The binding's own checks: tensors off the GPU are refused, never copied."""
    import torch
    q = torch.zeros(4, 2, 32)
    for call in (lambda: T.rel_attention(q, q, q, None, [0, 4]),
                 lambda: T.event_attention(q, q, q, [0, 4], [0, 1], [0, 4], [4]),
                 lambda: T.preference_loss(torch.zeros(4), torch.zeros(4, dtype=torch.int32), [0, 2, 4])):
        with pytest.raises(T.TxError) as e:
            call()
        assert e.value.code == T.TX_E_INVALID and "GPU" in str(e.value)
    for where in (([0, 4], [0, 1, 2], [0, 4], [4]), ([0, 4], [0, 1], [0, 4, 5], [4]), ([0, 4], [0, 1], [0, 4], [4, 4]),
                  ([0, 4], [1, 1], [0, 4], [4])):
        with pytest.raises(T.TxError):
            T.event_attention(q, q, q, *where)


@pytest.mark.parametrize("backward", [False, True])
def test_written_tensors_begin_apart(L, backward):
    at = {n: A + (i << 32) for i, n in enumerate(("q", "k", "v", "out", "dq", "dk", "dv"))}
    heads = lambda n: 2 if n in ("k", "v", "dk", "dv") else 4
    names = list(at) if backward else list(at)[:4]
    for w in ("dq", "dk", "dv") if backward else ("out",):
        for other in names:
            if other == w:
                continue
            t = {n: _rows(heads(n), data=at[other] if n == w else at[n]) for n in names}
            assert _rel(L, backward, **t) == T.TX_E_INVALID, (w, other)
            assert b"begins where" in L.tx_last_error()
    if backward:
        assert _pref(L, True) == T.TX_E_INVALID and b"begins where" in L.tx_last_error()


@pytest.mark.parametrize("backward", [False, True])
def test_calls_past_one_grid(L, backward):
    U = T.TX_E_UNSUPPORTED
    big = dict(q=_rows(65536, 32), out=_rows(65536, 32), k=_rows(1, 32), v=_rows(1, 32))
    if backward:
        big.update(dq=_rows(65536, 32), dk=_rows(1, 32), dv=_rows(1, 32))
    n = 300
    c = _cfg(H=65536, G=1, dh=32, R=0)
    if backward:  # (d_out of the helper has 4 heads of 64: rows that overlap may be read)
        assert _rel(L, True, cfg=c, off=np.arange(n + 1), lse_stride=n, **big) == U
    else:
        assert _rel(L, False, cfg=c, off=np.arange(n + 1), lse_stride=n, **big) == U
    assert b"one launch" in L.tx_last_error()
    c = _cfg(H=65536, G=1, dh=32, R=512)
    assert _rel(L, backward, cfg=c, off=(0, 5, 9), **big) == U and b"buckets" in L.tx_last_error()
    p = T.PreferenceConfig(T.TX_F32, 4, 0.1, 0.0)
    off = T._i64([0, 2, 5])
    assert L.tx_preference_workspace_bytes(ctypes.byref(p), (1 << 24) + 1, T._p(off, T.I64P)) == 0
    assert b"n_pairs" in L.tx_last_error()
