"""Argument checks of zipmoe_group_tokens, zipmoe_grouped_matmul, zipmoe_combine_rows and zipmoe_quantize_rows, which come
before anything is launched and so need no GPU (addresses here are never followed), and the oracle's own pins."""
import ctypes

import numpy as np
import pytest

from oracle import grouped
from paper_2601_21198_b200 import build

A = 1 << 20      # an aligned address that nobody reads


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def refused(zb, wanted, fn, *args, **kw):
    with pytest.raises(zb.ZipMoEError) as err:
        fn(*args, **kw)
    assert err.value.status == wanted, zb.zipmoe_status_string(err.value.status)


def test_group_refusals(zb):
    def call(ids=A, T=4, k=2, E=8, offsets=A, order=A, place=A, status=None):
        zb.zipmoe_group_tokens(ids, T, k, E, offsets, order, place, status)

    for kw in (dict(ids=None), dict(offsets=None), dict(order=None), dict(ids=A + 2), dict(offsets=A + 1), dict(order=A + 2),
               dict(place=A + 3), dict(status=A + 1)):
        refused(zb, zb.ERR_INVALID_ARG, call, **kw)
    for kw in (dict(E=0), dict(E=257), dict(k=0), dict(k=9), dict(T=1 << 28, k=8)):
        refused(zb, zb.ERR_UNSUPPORTED, call, **kw)


def test_grouped_matmul_refusals(zb):
    def weights(E=4, rows=64, cols=64, flags=0, even=1, table=None):
        return zb.GroupedWeightsStruct(E, rows, cols, flags, even, 0, table)

    def call(w=None, x=A, xp=64, xr=8, out=A, op=64, rows=8, offsets=A, order=None, k=0, rs=None, cs=None, flags=0, ws=None, n=0, status=None):
        zb.zipmoe_grouped_matmul(w or weights(), x, xp, xr, out, op, rows, offsets, order, k, rs, cs, flags, ws, n, status)

    for kw in (dict(x=None), dict(out=None), dict(xr=0), dict(xr=7), dict(xp=56), dict(op=63), dict(offsets=None), dict(order=A),
               dict(w=weights(even=0)), dict(w=weights(even=2)), dict(w=weights(flags=4)), dict(flags=1), dict(rs=A), dict(cs=A),
               dict(w=weights(flags=2), rs=A), dict(w=weights(flags=2), cs=A), dict(x=A + 8), dict(out=A + 1), dict(out=A + 2, flags=4),
               dict(w=weights(even=0, table=A + 32)), dict(offsets=A + 2), dict(order=A + 1, k=1), dict(status=A + 2)):
        refused(zb, zb.ERR_INVALID_ARG, call, **kw)
    for kw in (dict(w=weights(E=0)), dict(w=weights(E=257)), dict(w=weights(rows=0)), dict(w=weights(cols=0)), dict(w=weights(cols=60)),
               dict(w=weights(cols=65544), xp=65544), dict(w=weights(cols=72, flags=2), xp=80, rs=A, cs=A), dict(xp=68), dict(order=A, k=9),
               dict(w=weights(rows=(1 << 20) + 1), op=1 << 21), dict(rows=(1 << 30) + 1), dict(xr=(1 << 30) + 1)):
        refused(zb, zb.ERR_UNSUPPORTED, call, **kw)
    call(rows=0)
    # gathered rows need room where there are many
    big = weights(rows=4096, cols=4096)
    need = zb.zipmoe_grouped_workspace_bytes(big, 10000, True)
    assert need == 10000 * 4096 * 2 and zb.zipmoe_grouped_workspace_bytes(big, 10000, False) == 0
    assert zb.zipmoe_grouped_workspace_bytes(big, 1, True) == 0
    many = dict(w=big, xp=4096, op=4096, rows=10000, xr=10000, order=A, k=1)
    refused(zb, zb.ERR_INVALID_ARG, call, ws=None, n=need, **many)
    refused(zb, zb.ERR_INVALID_ARG, call, ws=A + 8, n=need, **many)
    refused(zb, zb.ERR_BUFFER_TOO_SMALL, call, ws=A, n=need - 1, **many)


def test_plan_refusals(zb):
    def plan(addresses, E=2, rows=64, cols=128, flags=0, table=np.zeros(1024, np.uint8)):
        ptrs = (ctypes.c_void_p * len(addresses))(*addresses)
        out = ctypes.byref(zb.GroupedWeightsStruct())
        return zb._lib.zipmoe_grouped_weights_plan(ptrs, E, rows, cols, flags, None if table is None else table.ctypes.data, out)

    assert plan([A, None]) == zb.ERR_INVALID_ARG
    assert plan([A, A + 8]) == zb.ERR_INVALID_ARG
    assert plan([A, A, A, None], flags=zb.GROUPED_PAIR) == zb.ERR_INVALID_ARG
    assert plan([A, A], table=None) == zb.ERR_INVALID_ARG
    assert plan([A, A], flags=zb.GROUPED_F32) == zb.ERR_INVALID_ARG
    for kw in (dict(E=0), dict(E=257), dict(rows=0), dict(cols=12), dict(cols=65544), dict(cols=8, flags=zb.GROUPED_INT8)):
        assert plan([A, A], **kw) == zb.ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        zb.zipmoe_grouped_weights_plan([A], 2, 64, 64)
    with pytest.raises(ValueError):
        zb.zipmoe_grouped_weights_plan([A, A], 2, 64, 64, zb.GROUPED_PAIR)


def test_combine_and_quantize_refusals(zb):
    def combine(y=A, yp=64, rows=8, place=A, w=A, T=4, k=2, cols=64, out=A, op=64, flags=0, status=None):
        zb.zipmoe_combine_rows(y, yp, rows, place, w, T, k, cols, out, op, flags, status)

    for kw in (dict(y=None), dict(place=None), dict(out=None), dict(yp=63), dict(op=63), dict(y=A + 1), dict(y=A + 2, flags=4),
               dict(out=A + 1), dict(place=A + 2), dict(w=A + 1), dict(status=A + 2), dict(flags=1)):
        refused(zb, zb.ERR_INVALID_ARG, combine, **kw)
    for kw in (dict(k=0), dict(k=9), dict(cols=0), dict(cols=(1 << 20) + 1, yp=1 << 21, op=1 << 21), dict(T=1 << 28, k=8)):
        refused(zb, zb.ERR_UNSUPPORTED, combine, **kw)
    combine(T=0)

    def quantize(x=A, xp=64, rows=4, cols=64, q=A, qp=64, s=A):
        zb.zipmoe_quantize_rows(x, xp, rows, cols, q, qp, s)

    for kw in (dict(x=None), dict(q=None), dict(s=None), dict(xp=63), dict(qp=63), dict(x=A + 1), dict(s=A + 2)):
        refused(zb, zb.ERR_INVALID_ARG, quantize, **kw)
    for kw in (dict(cols=0), dict(cols=65537, xp=70000, qp=70000), dict(rows=(1 << 30) + 1)):
        refused(zb, zb.ERR_UNSUPPORTED, quantize, **kw)
    quantize(rows=0)


def test_linear_refusals(zb):
    def weights(E=1, rows=64, cols=64, flags=2, even=1):
        return zb.GroupedWeightsStruct(E, rows, cols, flags, even, 0, None)

    need = zb.zipmoe_linear_int8_workspace_bytes(weights(), 8)
    assert need == 8 * 64 + 8 * 4

    def call(w=None, x=A, xp=64, rows=8, cs=A, out=A, op=64, ws=A, n=need, flags=0, status=None):
        zb.zipmoe_linear_int8(w or weights(), x, xp, rows, cs, out, op, ws, n, flags, status)

    for kw in (dict(x=None), dict(cs=None), dict(out=None), dict(ws=None), dict(xp=63), dict(op=63), dict(x=A + 1), dict(cs=A + 2),
               dict(out=A + 1), dict(out=A + 2, flags=4), dict(ws=A + 8), dict(flags=1), dict(status=A + 1), dict(w=weights(E=2)),
               dict(w=weights(flags=0)), dict(w=weights(flags=3)), dict(w=weights(even=0))):
        refused(zb, zb.ERR_INVALID_ARG, call, **kw)
    for kw in (dict(w=weights(rows=0)), dict(w=weights(cols=72), xp=72), dict(rows=(1 << 30) + 1)):
        refused(zb, zb.ERR_UNSUPPORTED, call, **kw)
    refused(zb, zb.ERR_BUFFER_TOO_SMALL, call, n=need - 1)
    call(rows=0)


def test_oracle_lists():
    ids = np.array([[1, 0], [-1, 1], [2, 2], [0, -7]])
    offsets, order, place = grouped.group(ids, 4)
    assert offsets.tolist() == [0, 2, 4, 6, 6] and order.tolist() == [1, 6, 0, 3, 4, 5]
    assert place.tolist() == [[2, 0], [-1, 3], [4, 5], [1, -1]]


def test_oracle_products_and_sums():
    rng = np.random.default_rng(0)
    ids = np.array([[1, 0], [1, -1], [0, 1]])
    x, w = rng.standard_normal((3, 5)), [rng.standard_normal((4, 5)) for _ in range(2)]
    wt = rng.standard_normal((3, 2))
    offsets, order, place = grouped.group(ids, 2)
    y = grouped.products(x, order // 2, offsets, w)
    out = grouped.combine(y, place, wt)
    for t in range(3):
        want = sum(wt[t, j] * (w[ids[t, j]] @ x[t]) for j in range(2) if ids[t, j] >= 0)
        assert np.allclose(out[t], want)


def test_oracle_quantize():
    x = np.array([[1.0, -2.0, 0.5, 0.0], [0.0, 0.0, 0.0, 0.0], [np.inf, 1.0, 0.0, 0.0], [3.0, np.nan, 0.0, 1.0]])
    q, s = grouped.quantize(x)
    assert q[0].tolist() == [64, -127, 32, 0]          # 63.5 -> 64 and 31.75 -> 32
    assert not q[1:].any() and s[0] == 2 / 127 and s[1] == 0 and np.isnan(s[2:]).all()
