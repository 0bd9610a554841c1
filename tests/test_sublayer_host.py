"""Argument checks of zipmoe_add_rmsnorm, zipmoe_route and zipmoe_expert_ffn, which come before anything is launched and
so need no GPU (addresses here are never followed), and the oracle's own pins."""
import ctypes

import numpy as np
import pytest

from oracle import sublayer
from paper_2601_21198_b200 import build

A = 1 << 20      # an aligned address that nobody reads


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def refused(zb, status, fn, *args, **kw):
    with pytest.raises(zb.ZipMoEError) as err:
        fn(*args, **kw)
    assert err.value.status == status, zb.zipmoe_status_string(err.value.status)


def test_norm_refusals(zb):
    def call(x=A, xp=64, r=A, rp=64, ro=A, rop=64, w=A, rows=4, cols=64, eps=1e-6, out=A, q=None, op=64, s=None, group=0, flags=0):
        zb.zipmoe_add_rmsnorm(x, xp, r, rp, ro, rop, w, rows, cols, eps, out, q, op, s, group, flags)

    inv, uns = zb.ERR_INVALID_ARG, zb.ERR_UNSUPPORTED
    for kw in (dict(x=None), dict(w=None), dict(out=None), dict(cols=0), dict(xp=63), dict(rp=63), dict(rop=63), dict(op=63),
               dict(r=None), dict(q=A), dict(s=A), dict(flags=2), dict(eps=-1.0), dict(eps=float("nan")), dict(x=A + 1),
               dict(r=A + 2, flags=1), dict(q=A, s=A + 2)):
        refused(zb, inv, call, **kw)
    refused(zb, uns, call, cols=32769, xp=40000, rp=40000, rop=40000, op=40000)
    refused(zb, uns, call, q=A, s=A, group=48)
    call(rows=0)


def test_route_refusals(zb):
    def call(x=A, T=4, pitch=64, g=A, E=16, H=64, b=None, k=2, flags=0, ids=A, w=A, logits=None):
        zb.zipmoe_route(x, T, pitch, g, E, H, b, k, flags, ids, w, logits)

    inv, uns = zb.ERR_INVALID_ARG, zb.ERR_UNSUPPORTED
    for kw in (dict(x=None), dict(g=None), dict(ids=None), dict(w=None), dict(flags=2), dict(pitch=56), dict(x=A + 8), dict(g=A + 2),
               dict(ids=A + 1), dict(w=A + 2), dict(b=A + 1), dict(logits=A + 1)):
        refused(zb, inv, call, **kw)
    for kw in (dict(E=0), dict(E=257), dict(k=0), dict(k=9), dict(k=5, E=4), dict(H=0), dict(H=60), dict(H=32776, pitch=32776),
               dict(pitch=68)):
        refused(zb, uns, call, **kw)
    call(T=0)


def test_expert_ffn_refusals(zb):
    def struct(E=4, H=64, I=128, table=A):
        return zb.ResidentExpertsStruct(E, H, I, 0, table)

    need = zb.zipmoe_expert_ffn_workspace_bytes(8, 2, struct())
    assert need > 0

    def call(x=A, T=8, ids=A, w=A, k=2, ex=None, out=A, ws=A, n=need):
        zb.zipmoe_expert_ffn(x, T, ids, w, k, ex or struct(), out, ws, n)

    inv, uns = zb.ERR_INVALID_ARG, zb.ERR_UNSUPPORTED
    for kw in (dict(x=None), dict(ids=None), dict(out=None), dict(ws=None), dict(ex=struct(table=None)), dict(x=A + 8),
               dict(out=A + 2), dict(ws=A + 4), dict(ex=struct(table=A + 32)), dict(ids=A + 2), dict(w=A + 1)):
        refused(zb, inv, call, **kw)
    for kw in (dict(T=257), dict(k=0), dict(k=9), dict(ex=struct(E=0)), dict(ex=struct(E=257)), dict(ex=struct(H=60)),
               dict(ex=struct(I=4)), dict(ex=struct(H=0)), dict(ex=struct(I=32776))):
        refused(zb, uns, call, **kw)
    refused(zb, zb.ERR_BUFFER_TOO_SMALL, call, n=need - 1)
    call(T=0)
    # more tokens, more choices, larger experts: never less scratch
    sizes = [zb.zipmoe_expert_ffn_workspace_bytes(T, 2, struct(H=1024, I=2048)) for T in (1, 2, 16, 64, 65, 256)]
    assert sizes == sorted(sizes)


def test_resident_plan_refusals(zb):
    lib = zb._lib
    table = np.zeros(3 * 2 * zb.RESIDENT_ENTRY_BYTES, np.uint8)

    def plan(addresses, E=2, H=64, I=128, out=table):
        ptrs = (ctypes.c_void_p * len(addresses))(*addresses)
        experts = ctypes.byref(zb.ResidentExpertsStruct())
        return lib.zipmoe_resident_experts_plan(ptrs, E, H, I, None if out is None else out.ctypes.data, experts)

    assert plan([A] * 5 + [None]) == zb.ERR_INVALID_ARG
    assert plan([A] * 5 + [A + 8]) == zb.ERR_INVALID_ARG
    assert plan([A] * 6, out=None) == zb.ERR_INVALID_ARG
    for kw in (dict(E=0), dict(E=257), dict(H=12), dict(I=0), dict(H=32776)):
        assert plan([A] * 6, **kw) == zb.ERR_UNSUPPORTED
    with pytest.raises(ValueError):
        zb.zipmoe_resident_experts_plan([A] * 5, 2, 64, 128)


def test_oracle_norm_has_unit_rms():
    rng = np.random.default_rng(0)
    x, r = rng.standard_normal((5, 300)), 4 * rng.standard_normal((5, 300))
    h, y = sublayer.add_rmsnorm(x, r, np.ones(300), 0.0)
    assert np.allclose(h, x + r) and np.allclose((y * y).mean(axis=1), 1.0)
    s = sublayer.group_scales(y, 128)
    assert s.shape == (5, 3) and np.allclose(s.max(axis=1), np.abs(y).max(axis=1) / 448)


def test_oracle_e4m3_table():
    v = sublayer.e4m3_to_f64(np.arange(256))
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[0x38] == 1.0 and v[0x7E] == 448.0 and v[0xFE] == -448.0
    assert np.isnan(v[0x7F]) and np.isnan(v[0xFF]) and (np.diff(v[:0x7F]) > 0).all()


def test_oracle_choice():
    l = np.array([[1.0, 3.0, 3.0, -np.inf, 2.0], [-np.inf] * 5, [-np.inf, 5.0, -np.inf, -np.inf, -np.inf]])
    assert sublayer.choose(l, 3).tolist() == [[1, 2, 4], [-1, -1, -1], [1, -1, -1]]
    w = sublayer.weights_of(l, sublayer.choose(l, 3))
    assert np.allclose(w.sum(axis=1), [1, 0, 1]) and w[0, 0] == w[0, 1]
    assert sublayer.weights_of(l, sublayer.choose(l, 3), renormalise=False)[0].sum() < 1
