"""Refusals of softmax attention and AdamW, without a GPU: every bad argument is answered with its status and a text before the device is used."""
import os

import numpy as np
import pytest

from paper_2309_03523_amd import binding

OK, INVALID, UNSUPPORTED = 0, 1, 4
Q, K, V, O, DO, DQ, DK, DV, LSE, BIAS, MAP, WS, DB = (0x10000000 * i for i in range(1, 14))      # aligned and far apart: never read


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return binding.load()


def _text(lib):
    return lib.dgc_last_error(None).decode()


COMMON = dict(Tq=40, Tk=40, N=5, heads=4, kv=2, d=16, dtype=0, causal=1, scale=0.25, first=None, lengths=None, keep=None, bias=BIAS, map=MAP, buckets=8, reach=12)
SHAPE = dict(qt=5 * 64, qn=64, kt=5 * 32, kn=32)
BAD = (dict(Tq=41), dict(Tq=-1), dict(Tk=1 << 31), dict(N=-1), dict(heads=0), dict(heads=3), dict(kv=0), dict(kv=3), dict(heads=2048), dict(d=12), dict(d=0), dict(d=136),
       dict(dtype=2), dict(dtype=-1), dict(buckets=257), dict(buckets=-1), dict(reach=1025), dict(reach=-1), dict(buckets=0), dict(bias=None), dict(map=None),
       dict(bias=None, map=None), dict(bias=BIAS + 2), dict(first=1), dict(lengths=3), dict(q=None), dict(k=None), dict(v=None), dict(o=None), dict(q=Q + 8), dict(k=K + 4),
       dict(qt=318), dict(qn=66), dict(kt=-160), dict(kn=-32), dict(qt=1 << 62), dict(lse=LSE + 1))


def _forward(lib, **kw):
    a = {**dict(q=Q, **SHAPE, k=K, v=V, o=O, lse=None, ws=None, ws_bytes=0), **COMMON, **kw}
    a.setdefault("ot", a["qt"]), a.setdefault("on", a["qn"])
    return lib.dgc_attn_forward(a["q"], a["qt"], a["qn"], a["k"], a["kt"], a["kn"], a["v"], a["kt"], a["kn"], a["Tq"], a["Tk"], a["N"], a["heads"], a["kv"], a["d"],
                                a["dtype"], a["causal"], a["scale"], a["first"], a["lengths"], a["keep"], a["bias"], a["map"], a["buckets"], a["reach"], a["o"],
                                a["ot"], a["on"], a["lse"], a["ws"], a["ws_bytes"], None)


def _backward(lib, **kw):
    a = {**dict(q=Q, **SHAPE, k=K, v=V, o=O, lse=LSE, go=DO, dq=DQ, dk=DK, dv=DV, db=DB, ws=WS, ws_bytes=1 << 24), **COMMON, **kw}
    for n, m in (("ot", "qt"), ("on", "qn"), ("dqt", "qt"), ("dqn", "qn"), ("dkt", "kt"), ("dkn", "kn")):
        a.setdefault(n, a[m])
    return lib.dgc_attn_backward(a["q"], a["qt"], a["qn"], a["k"], a["kt"], a["kn"], a["v"], a["kt"], a["kn"], a["o"], a["ot"], a["on"], a["lse"], a["go"], a["ot"],
                                 a["on"], a["Tq"], a["Tk"], a["N"], a["heads"], a["kv"], a["d"], a["dtype"], a["causal"], a["scale"], a["first"], a["lengths"],
                                 a["keep"], a["bias"], a["map"], a["buckets"], a["reach"], a["dq"], a["dqt"], a["dqn"], a["dk"], a["dkt"], a["dkn"], a["dv"],
                                 a["dkt"], a["dkn"], a["db"], a["ws"], a["ws_bytes"], None)


def test_attention_refusals(lib):
    few = dict(Tq=1, Tk=5000, kt=160, kn=32)
    need = lib.dgc_attn_workspace_bytes(1, 5000, 5, 4, 2, 16, 0, 1, 8, 12, 0)
    assert need > 0 and need % 16 == 0
    for kw in BAD + (dict(ot=32), dict(on=32), dict(o=Q), dict(o=K + 16), dict(o=Q + 32), dict(lse=Q), dict(lse=O), dict(lse=O + 64), dict(o=BIAS - 64),
                     few, dict(few, ws=WS, ws_bytes=need - 1), dict(few, ws=WS + 8, ws_bytes=need), dict(few, ws=O, ws_bytes=need), dict(few, ws=K + 160, ws_bytes=need),
                     dict(few, ws=MAP, ws_bytes=need)):
        assert _forward(lib, **kw) == INVALID, kw
        assert "attention" in _text(lib)
    assert _forward(lib, N=1 << 40) in (INVALID, UNSUPPORTED)
    for kw in (dict(N=0, q=None, k=None, v=None, o=None), dict(Tq=0, q=None, o=None), dict(Tq=0, Tk=0, q=None, k=None, v=None, o=None)):
        assert _forward(lib, **kw) == OK, _text(lib)
    for kw in BAD + (dict(lse=None), dict(db=DB + 2), dict(db=BIAS), dict(db=DQ), dict(dq=Q), dict(dk=K), dict(dv=V), dict(dq=DO), dict(dq=O), dict(dv=DK), dict(dk=DV + 16),
                     dict(dqt=32), dict(dkn=16), dict(dq=DQ + 4), dict(ws=None), dict(ws=WS + 4), dict(ws_bytes=16), dict(ws=LSE), dict(ws=DV), dict(dv=WS + 64),
                     dict(bias=None, map=None, buckets=0, reach=0), dict(go=None), dict(go=DO + 8)):
        assert _backward(lib, **kw) == INVALID, kw
        assert "attention" in _text(lib)
    for kw in (dict(N=1 << 25), dict(N=1 << 20, heads=64, kv=64, Tk=40), dict(N=1 << 17, Tq=1 << 20, Tk=1 << 20)):
        sizes = dict(dict(Tq=40, Tk=40, N=5, heads=4, kv=2), **kw)
        assert lib.dgc_attn_workspace_bytes(sizes["Tq"], sizes["Tk"], sizes["N"], sizes["heads"], sizes["kv"], 16, 0, 1, 0, 0, 1) < 0, kw


def test_columns_side_by_side_do_not_overlap(lib):
    """Queries, keys, values and their gradients as columns of one buffer each; a device is the next thing the call needs."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")
    side = dict(kv=4, qt=5 * 192, qn=192, kt=5 * 192, kn=192)
    assert _forward(lib, **side, k=Q + 256, v=Q + 512, ot=5 * 64, on=64) not in (OK, INVALID, UNSUPPORTED)
    assert _forward(lib, **side, k=Q + 256, v=Q + 512, o=Q + 256) == INVALID
    assert _backward(lib, **side, k=Q + 256, v=Q + 512, ot=5 * 64, on=64, dk=DQ + 256, dv=DQ + 512) not in (OK, INVALID, UNSUPPORTED)
    assert _backward(lib, **side, k=Q + 256, v=Q + 512, ot=5 * 64, on=64, dk=DQ + 240, dv=DQ + 512) == INVALID


def test_workspaces_grow_with_what_they_hold(lib):
    size = lambda Tq, Tk, N=3, heads=4, kv=2, d=32, back=1, buckets=8: lib.dgc_attn_workspace_bytes(Tq, Tk, N, heads, kv, d, 1, 1, buckets, 64 if buckets else 0, back)  # noqa: E731
    assert size(0, 50) > 0 and size(0, 0) == 0 and size(50, 50, N=0) == 0
    for Ts in ((1, 7, 40, 200, 5000), (1, 300, 1 << 20)):
        got = [size(T, T) for T in Ts]
        assert all(0 < a <= b for a, b in zip(got, got[1:]))
    assert size(100, 100) >= size(100, 100, buckets=0) >= 4 * 3 * 4 * 100
    for Tk in (1, 200, 5000, 1 << 20):
        assert 0 <= size(1, Tk, back=0) <= 4 * 3 * 4 * 34 * 1024 + 16
    for bad in (dict(N=-1), dict(heads=3), dict(d=20), dict(kv=0)):
        assert size(4, 4, **bad) < 0
    assert size(5, 4) < 0


def test_buckets_of_distance(lib):
    """Half of a side's buckets hold one distance each; the others begin at single (reach / single)^(k / rest) and the last holds what lies beyond."""
    for buckets, reach, causal in ((16, 32, True), (2, 1, True), (3, 1, True), (9, 1024, True), (256, 1024, True), (4, 1, False), (32, 128, False), (16, 8, True)):
        got = binding.attn_buckets(buckets, reach, causal=causal)
        assert got.dtype == np.uint8 and got.shape == (2 * reach + 1,) and got.max() < buckets
        side = buckets if causal else buckets // 2
        single = side // 2
        ahead, past = got[:reach][::-1], got[reach:]
        assert (ahead == 0).all() if causal else (ahead == past[1:] + side).all()
        assert (past[:single] == np.arange(single)).all() and (np.diff(past.astype(int)) >= 0).all() and past[reach] == (side - 1 if reach >= single else reach)
        for k in range(1, side - single):
            if reach <= single:
                break
            edge = single * (reach / single) ** (k / (side - single))      # a distance below the edge is in an earlier bucket, one above not
            x = np.arange(reach + 1)
            assert (past[x < edge - 1e-6] < single + k).all() and (past[x > edge + 1e-6] >= single + k).all()
    out = np.zeros(99, np.uint8)
    for args in ((1, 32, 1), (257, 32, 1), (16, 0, 1), (16, 1025, 1), (15, 32, 0), (2, 32, 0), (16, 7, 1), (32, 7, 0)):
        assert lib.dgc_attn_buckets(*args, out.ctypes.data) == INVALID, args
        assert "buckets" in _text(lib)
    assert lib.dgc_attn_buckets(16, 32, 1, None) == INVALID


def _tensor(**kw):
    a = dict(dict(p=Q, g=K, master=None, m=V, v=O, m_scale=None, v_scale=None, R=10, ldp=32, ldg=32, ldmaster=0, F=30, dtype=0, weight_decay=0.0), **kw)
    return binding.AdamwTensorT(**a)


def test_adamw_refusals(lib):
    import ctypes as ct

    def create(items, bits=32, n=None):
        h = ct.c_void_p()
        rc = lib.dgc_adamw_create((binding.AdamwTensorT * max(1, len(items)))(*items), len(items) if n is None else n, bits, ct.byref(h))
        assert rc == OK or not h.value
        return rc, h

    eight = dict(m_scale=DQ, v_scale=DK)
    for items, bits in (([_tensor(p=None)], 32), ([_tensor(g=None)], 32), ([_tensor(m=None)], 32), ([_tensor(v=None)], 32), ([_tensor(p=Q + 4)], 32), ([_tensor(ldp=29)], 32),
                        ([_tensor(ldp=31)], 32), ([_tensor(dtype=2)], 32), ([_tensor(R=-1)], 32), ([_tensor(F=-1)], 32), ([_tensor(weight_decay=-1.0)], 32),
                        ([_tensor(weight_decay=float("nan"))], 32), ([_tensor()], 16), ([_tensor()], 0), ([_tensor()], 8), ([_tensor(m_scale=DQ)], 8),
                        ([_tensor(master=DO, ldmaster=32)], 32),      # fp32 parameters are their own masters
                        ([_tensor(dtype=1, master=DO + 4, ldmaster=32)], 32), ([_tensor(dtype=1, master=DO, ldmaster=28)], 32), ([_tensor(dtype=1, ldp=36)], 32),
                        ([_tensor(g=Q)], 32), ([_tensor(m=Q)], 32), ([_tensor(v=V)], 32), ([_tensor(v=V + 64)], 32), ([_tensor(m=K)], 32),
                        ([_tensor(**dict(eight, v_scale=DQ))], 8), ([_tensor(**dict(eight, m_scale=V))], 8),
                        ([_tensor(), _tensor(p=DQ, g=DK, m=DV, v=LSE), _tensor(p=Q, g=BIAS, m=MAP, v=WS)], 32),
                        ([_tensor(), _tensor(p=DQ, g=DK, m=V + 32 * 40 - 16, v=LSE)], 32)):
        assert create(items, bits)[0] == INVALID, [{n: getattr(t, n) for n, _ in t._fields_} for t in items]
        assert "adamw" in _text(lib)
    assert create([_tensor()], n=-1)[0] == INVALID
    assert lib.dgc_adamw_create(None, 1, 32, ct.byref(ct.c_void_p())) == INVALID and lib.dgc_adamw_create(None, 0, 32, None) == INVALID
    assert create([_tensor(R=1 << 40)])[0] in (INVALID, UNSUPPORTED)
    # Nothing to step needs no device: an empty handle's steps are checked all the same.
    for items in ([], [_tensor(R=0, p=None, g=None, m=None, v=None)], [_tensor(F=0, p=None, g=None, m=None, v=None)]):
        rc, h = create(items)
        assert rc == OK, _text(lib)
        step = lambda lr=0.1, b1=0.9, b2=0.99, eps=1e-8, t=1, steps=None, at=None: lib.dgc_adamw_step(h, lr, b1, b2, eps, t, steps, at, None)  # noqa: E731
        assert step() == OK
        inf, nan = float("inf"), float("nan")
        for kw in (dict(lr=-1.0), dict(lr=inf), dict(lr=nan), dict(b1=1.0), dict(b1=-0.1), dict(b1=nan), dict(b2=1.0), dict(b2=nan), dict(eps=-1e-9), dict(eps=nan), dict(eps=inf),
                   dict(t=0), dict(t=-3), dict(at=WS), dict(steps=WS + 4), dict(steps=WS, at=LSE + 2)):
            assert step(**kw) == INVALID, kw
            assert "adamw" in _text(lib)
        lib.dgc_adamw_destroy(h)
    assert lib.dgc_adamw_step(None, 0.1, 0.9, 0.99, 1e-8, 1, None, None, None) == INVALID
    lib.dgc_adamw_destroy(None)


def test_the_optimizer_refuses_before_a_device_is_used():
    import torch
    from paper_2309_03523_amd.optimizer import AdamW
    p, g = torch.zeros(3, 8), torch.zeros(3, 8)
    for args, kw in ((([], []), {}), (([p], []), {}), (([p], [g]), dict(bits=16)), (([p], [g]), dict(betas=(1.0, 0.9))), (([p], [g]), dict(eps=-1.0)),
                     (([p], [g]), dict(steps=-1)), (([p], [g]), dict(weight_decay=-0.1)), (([p], [g]), dict(weight_decay=[0.1, 0.1])), (([p], [g]), dict(states=[])),
                     (([p], [g]), dict(masters=[])), (([p], [g]), {})):      # the last: not on a device
        with pytest.raises(ValueError):
            AdamW(*args, **kw)
