"""The grouped products, the lists they go by and the weighted sums on the GPU against the fp64 oracle.

Where operands lie on coarse grids every product and partial sum is exact in fp32, whatever its order, so a single product has
to be the correctly rounded value, bit for bit.  The gated activation adds the fp32 exponential (2 units of 2^-23, and |g| of
them from its argument), a division and two products: (8 + 2 |g|) * 2^-23 of the value, and half a step of bf16.  The
weighted sums are k fp32 additions: (k + 1) * 2^-24 of the sum of the magnitudes, and half a step."""
import numpy as np
import pytest

from oracle import grouped
from oracle.ffn import bf16_to_f64
from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


@pytest.fixture(params=[1, 2], ids=["few", "many"])
def kernel(zb, request):
    """Either kernel on every size: which one a call takes is a matter of speed."""
    zb.zipmoe_test_grouped_kernel(request.param)
    yield request.param
    zb.zipmoe_test_grouped_kernel(0)


def half_step(v):
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - 8)


def coarse(shape, seed, step):
    """Whole multiples of `step`, at most 8 of them: products of two such and sums of 2^17 of those are exact in fp32."""
    rng = np.random.default_rng(seed)
    return np.clip(np.rint(rng.standard_normal(shape) * 2.5), -8, 8) * step


def bf16(a):
    import torch
    return torch.from_numpy(np.asarray(a, np.float32)).cuda().to(torch.bfloat16)


def host(t):
    return t.float().cpu().numpy().astype(np.float64)


def routing(T, k, E, seed, dropped=0.0, only=None):
    """ids [T, k]: a token's experts are distinct where there are enough; `only`: the experts that may be chosen."""
    rng = np.random.default_rng(seed)
    pool = np.arange(E) if only is None else np.asarray(only)
    ids = np.stack([rng.permutation(pool)[:k] if len(pool) >= k else rng.choice(pool, k) for _ in range(T)]).astype(np.int32)
    ids[rng.random((T, k)) < dropped] = -1
    return ids


def gpu(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


# ---- lists ------------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,k,E", [(1, 1, 1), (1, 8, 8), (3, 2, 5), (64, 2, 8), (127, 4, 60), (1000, 1, 256), (777, 6, 64), (2049, 8, 255),
                                   (8192, 6, 64), (16411, 8, 33)])
@pytest.mark.parametrize("dropped", [0.0, 0.3, 1.0])
def test_lists(zb, T, k, E, dropped):
    import torch
    ids = routing(T, k, E, T + k, dropped)
    order = torch.full((T * k,), -77, dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    g = zb.group_tokens(gpu(ids), E, order=order, status=status)
    offsets, want, place = grouped.group(ids, E)
    assert np.array_equal(g.offsets.cpu().numpy(), offsets)
    assert np.array_equal(g.order.cpu().numpy()[:want.size], want)
    assert (g.order.cpu().numpy()[want.size:] == -77).all()          # behind the last group: left as it was
    assert np.array_equal(g.place.cpu().numpy(), place) and int(status.item()) == 0


@pytest.mark.parametrize("T,k,E", [(40000, 8, 64), (70001, 5, 256), (131073, 1, 3)])
def test_lists_of_many_choices(zb, T, k, E):
    """More than the warps of the largest cluster hold in registers."""
    ids = np.random.default_rng(T).integers(-1, E, (T, k)).astype(np.int32)
    g = zb.group_tokens(gpu(ids), E)
    offsets, want, place = grouped.group(ids, E)
    assert np.array_equal(g.offsets.cpu().numpy(), offsets)
    assert np.array_equal(g.order.cpu().numpy()[:want.size], want) and np.array_equal(g.place.cpu().numpy(), place)


def test_lists_of_no_tokens_repeated_and_wrong_ids(zb):
    import torch
    g = zb.group_tokens(torch.empty(0, 3, dtype=torch.int32, device="cuda"), 7)
    assert not g.offsets.any() and g.offsets.shape == (8,) and g.rows == 0
    ids = np.array([[2, 2], [2, 9], [-5, 0], [2**31 - 1, -2**31]], np.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    g = zb.group_tokens(gpu(ids), 3, status=status)
    assert g.offsets.tolist() == [0, 1, 1, 4] and g.order.tolist()[:4] == [5, 0, 1, 2]
    assert g.place.tolist() == [[1, 2], [3, -1], [-1, 0], [-1, -1]] and int(status.item()) == 1


# ---- products ---------------------------------------------------------------------------------------------------
SHAPES = [(1, 1, 1, 8, 8), (1, 2, 2, 64, 64), (5, 3, 2, 72, 40), (40, 1, 1, 136, 200), (64, 4, 2, 2048, 128), (65, 4, 1, 256, 129), (100, 7, 3, 520, 257),
          (300, 2, 1, 192, 384), (777, 60, 4, 264, 136), (30, 256, 8, 64, 72), (1100, 3, 2, 1032, 520), (2500, 8, 2, 128, 264),
          (33, 1, 1, 320, 256), (257, 1, 1, 384, 513), (512, 1, 1, 448, 512), (513, 1, 1, 512, 768), (600, 2, 1, 64, 700), (256, 1, 1, 3000, 8)]


@pytest.mark.parametrize("T,E,k,K,N", SHAPES)
@pytest.mark.parametrize("gather", [False, True])
def test_product_is_the_rounded_sum(zb, kernel, T, E, k, K, N, gather):
    import torch
    ids = routing(T, k, E, T, dropped=0.1 if T > 4 else 0.0)
    g = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    x, w = coarse((T if gather else T * k, K), 1, 1 / 16), coarse((E, N, K), 2, 1 / 64)
    m = zb.GroupedMatrix(list(bf16(w)))
    assert m.struct.even
    want = grouped.products(x, order // k if gather else np.arange(len(order)), offsets, w)
    for dtype in (torch.bfloat16, torch.float32):
        out = torch.full((T * k, N), 7.0, dtype=dtype, device="cuda")
        assert m.product(bf16(x), g, gather=gather, out=out) is out
        assert torch.equal(out[:len(order)], torch.from_numpy(want).cuda().to(dtype))
        assert (out[len(order):] == 7.0).all() and int(m.status.item()) == 0


def check_gated(h, first, second):
    want = grouped.gated(first, second)
    bound = half_step(want) * (1 + 2.0 ** -10) + np.abs(want) * (8 + 2 * np.abs(first)) * 2.0 ** -23 + 1e-30
    assert (np.abs(host(h) - want) <= bound).all(), float((np.abs(host(h) - want) / bound).max())


@pytest.mark.parametrize("T,E,k,K,N", SHAPES)
@pytest.mark.parametrize("gather", [False, True])
def test_pairs(zb, kernel, T, E, k, K, N, gather):
    import torch
    ids = routing(T, k, E, T + 1, dropped=0.1 if T > 4 else 0.0)
    g = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    x, w1, w3 = coarse((T if gather else T * k, K), 3, 1 / 16), coarse((E, N, K), 4, 1 / 64), coarse((E, N, K), 5, 1 / 64)
    m = zb.GroupedMatrix(list(bf16(w1)), up=list(bf16(w3)))
    src = order // k if gather else np.arange(len(order))
    out = torch.full((T * k, N), 7.0, dtype=torch.bfloat16, device="cuda")
    m.product(bf16(x), g, gather=gather, out=out)
    check_gated(out[:len(order)], grouped.products(x, src, offsets, w1), grouped.products(x, src, offsets, w3))
    assert (out[len(order):] == 7.0).all() and int(m.status.item()) == 0


@pytest.mark.parametrize("T,E,k,K,N", [(3, 2, 1, 32, 8), (70, 3, 2, 144, 136), (600, 5, 2, 1040, 264), (2500, 3, 1, 128, 130),
                                       (300, 1, 1, 896, 520)])
@pytest.mark.parametrize("pair", [False, True])
@pytest.mark.parametrize("gather", [False, True])
def test_int8_groups(zb, kernel, T, E, k, K, N, pair, gather):
    import torch
    rng = np.random.default_rng(K)
    ids = routing(T, k, E, T + 2, dropped=0.1 if T > 4 else 0.0)
    g = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    rows = T if gather else T * k
    x, w = rng.integers(-128, 128, (rows, K), dtype=np.int8), rng.integers(-128, 128, (2, E, N, K), dtype=np.int8)
    sx, sw = (rng.random(rows) / 64 + 1e-3).astype(np.float32), (rng.random((2, E, N)) / 64 + 1e-3).astype(np.float32)
    src = order // k if gather else np.arange(len(order))
    m = zb.GroupedMatrix(list(gpu(w[0])), up=list(gpu(w[1])) if pair else None, scales=gpu(sw[0]), up_scales=gpu(sw[1]) if pair else None)
    of = np.repeat(np.arange(E), np.diff(offsets))
    # the integers are exact; their conversion and the two scales are fp32
    acc = [grouped.products(x.astype(np.float64), src, offsets, w[j].astype(np.float64)) for j in range(2)]
    scaled = [(a.astype(np.float32) * sx[src][:, None]).astype(np.float32) * s[of] for a, s in zip(acc, sw)]
    out = torch.full((T * k, N), 7.0, device="cuda")
    m.product(gpu(x), g, gather=gather, row_scales=gpu(sx), out=out)
    half = m.product(gpu(x), g, gather=gather, row_scales=gpu(sx))
    assert half.dtype == torch.bfloat16 and torch.equal(out[:len(order)].to(torch.bfloat16), half[:len(order)])
    if pair:
        want = grouped.gated(*[s.astype(np.float64) for s in scaled])
        bound = np.abs(want) * (8 + 2 * np.abs(scaled[0])) * 2.0 ** -23 + 1e-30
        assert (np.abs(host(out[:len(order)]) - want) <= bound).all()
    else:
        assert np.array_equal(out[:len(order)].cpu().numpy(), scaled[0])
    assert (out[len(order):] == 7.0).all() and int(m.status.item()) == 0


def test_one_group_without_lists(zb, kernel):
    import torch
    x, w = coarse((333, 200), 6, 1 / 16), coarse((72, 200), 7, 1 / 64)
    m = zb.GroupedMatrix([bf16(w)])
    assert torch.equal(m.product(bf16(x)), torch.from_numpy(x @ w.T).cuda().to(torch.bfloat16))
    assert m.product(bf16(x)[:0]).shape == (0, 72)
    bits = m.product(bf16(x).view(torch.int16))                        # int16 patterns in, int16 patterns out
    assert bits.dtype == torch.int16 and torch.equal(bits.view(torch.bfloat16), m.product(bf16(x)))


@pytest.mark.parametrize("T", [6, 500])
@pytest.mark.parametrize("pair", [False, True])
def test_strides_and_scattered_weights(zb, kernel, T, pair):
    """Rows of x and out that lie apart (out even off any vector's boundary), weights in no order, int16 patterns."""
    import torch
    E, k, K, N = 5, 2, 136, 90
    ids = routing(T, k, E, 9, dropped=0.2)
    g = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    x, w = coarse((T, K), 8, 1 / 16), coarse((2, E, N, K), 9, 1 / 64)
    apart = [[bf16(m) for m in reversed(w[j])][::-1] for j in range(2)]
    apart[0][1], apart[1][1] = bf16(w[0, 1]), bf16(w[1, 1])
    m = zb.GroupedMatrix(apart[0], up=apart[1] if pair else None)
    wide_x = torch.full((T, K + 24), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide_x[:, 8:8 + K] = bf16(x)
    wide_out = torch.full((T * k, N + 11), 7.0, dtype=torch.bfloat16, device="cuda")
    out = wide_out[:, 3:3 + N]
    m.product(wide_x[:, 8:8 + K], g, gather=True, out=out)
    first = grouped.products(x, order // k, offsets, w[0])
    if pair:
        check_gated(out[:len(order)], first, grouped.products(x, order // k, offsets, w[1]))
    else:
        assert torch.equal(out[:len(order)], torch.from_numpy(first).cuda().to(torch.bfloat16))
    wide_out[:len(order), 3:3 + N] = 7.0
    assert (wide_out == 7.0).all()


@pytest.mark.parametrize("T", [20, 700])
def test_empty_and_lopsided_groups(zb, kernel, T):
    """All tokens on one expert, the others without any; rows of other groups and behind the last hold NaN and infinities."""
    import torch
    E, K, N = 9, 128, 140
    x, w = coarse((T, K), 10, 1 / 16), coarse((E, N, K), 11, 1 / 64)
    m = zb.GroupedMatrix(list(bf16(w)))
    for only in ([0], [8], [4], [0, 8]):
        ids = routing(T, 1, E, 12, only=only)
        ids[::7] = -1
        g = zb.group_tokens(gpu(ids), E)
        offsets, order, _ = grouped.group(ids, E)
        rows = torch.full((T, K), float("nan"), dtype=torch.bfloat16, device="cuda")
        rows[:len(order)] = bf16(x)[:len(order)]
        out = m.product(rows, g)
        want = grouped.products(x, np.arange(T), offsets, w)
        assert torch.equal(out[:len(order)], torch.from_numpy(want).cuda().to(torch.bfloat16))
    # a token of NaN spoils its own rows only
    ids = routing(T, 2, E, 13)
    g = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    y = bf16(x)
    y[3] = float("nan")
    y[5, 0] = float("inf")
    out = m.product(y, g, gather=True)
    spoilt = np.isin(order // 2, [3, 5])
    want = grouped.products(x, order // 2, offsets, w)
    assert torch.equal(out[gpu(~spoilt)], torch.from_numpy(want[~spoilt]).cuda().to(torch.bfloat16))
    assert out[gpu(order // 2 == 3)].isnan().all() and not out[gpu(order // 2 == 5)].isfinite().any(dim=0).all()


@pytest.mark.parametrize("rows", [10, 600])
def test_wrong_lists_are_reported(zb, kernel, rows):
    """Offsets out of order or past the end leave everything as it was, a row that is nowhere counts as zeros."""
    import torch
    E, K, N = 3, 64, 64
    x, w = coarse((rows, K), 14, 1 / 16), coarse((E, N, K), 15, 1 / 64)
    m = zb.GroupedMatrix(list(bf16(w)))
    third = rows // 3
    for offsets in ([0, third, 2 * third, rows + 1], [0, 2 * third, third, rows], [-1, third, third, rows]):
        g = zb.TokenGroups(gpu(np.array(offsets, np.int32)), gpu(np.arange(rows, dtype=np.int32)), torch.zeros(rows, 1, dtype=torch.int32, device="cuda"), E)
        out = torch.full((rows, N), 7.0, dtype=torch.bfloat16, device="cuda")
        m.product(bf16(x), g, out=out)
        assert int(m.status.item()) == 1 and (out == 7.0).all()
        m.status.zero_()
    order = np.arange(rows, dtype=np.int32)
    order[2], order[7] = -3, rows
    g = zb.TokenGroups(gpu(np.array([0, third, 2 * third, rows], np.int32)), gpu(order), torch.zeros(rows, 1, dtype=torch.int32, device="cuda"), E)
    out = m.product(bf16(x), g, gather=True)
    assert int(m.status.item()) == 1 and not out[2].any() and not out[7].any()
    keep = [r for r in range(third) if r not in (2, 7)]
    assert torch.equal(out[keep].cpu(), torch.from_numpy(x[keep] @ w[0].T).to(torch.bfloat16))


@pytest.mark.parametrize("T", [9, 500])
def test_products_of_some_of_the_experts(zb, kernel, T):
    """Part of the offsets, whose first is not 0: other experts' rows are neither read nor written, nor what `order` says there."""
    import torch
    E, k, K, N, lo, hi = 8, 2, 136, 96, 2, 6
    x, w = coarse((T, K), 21, 1 / 16), coarse((E, N, K), 22, 1 / 64)
    ids = routing(T, k, E, 23, dropped=0.1)
    g = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    begin, end = int(offsets[lo]), int(offsets[hi])
    assert 0 < begin < end < len(order)
    g.order[:begin] = -5
    g.order[end:] = 1 << 30
    m = zb.GroupedMatrix(list(bf16(w[lo:hi])))
    out = torch.full((T * k, N), 7.0, dtype=torch.bfloat16, device="cuda")
    m.product(bf16(x), zb.TokenGroups(g.offsets[lo:hi + 1], g.order, g.place, hi - lo), gather=True, out=out)
    want = grouped.products(x, order // k, offsets, w)[begin:end]
    assert int(m.status.item()) == 0 and (out[:begin] == 7.0).all() and (out[end:] == 7.0).all()
    assert torch.equal(out[begin:end], torch.from_numpy(want).cuda().to(torch.bfloat16))


# ---- weighted sums ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("T,k,cols", [(1, 1, 8), (1, 8, 4096), (5, 2, 100), (64, 3, 1408), (33, 6, 30), (700, 4, 264), (70000, 1, 8)])
@pytest.mark.parametrize("f32", [False, True])
def test_combine(zb, T, k, cols, f32):
    import torch
    rng = np.random.default_rng(T)
    E = 9
    ids = routing(T, k, E, T, dropped=0.2)
    ids[0] = -1
    g = zb.group_tokens(gpu(ids), E)
    _, order, place = grouped.group(ids, E)
    y = torch.from_numpy(rng.standard_normal((T * k, cols)).astype(np.float32)).cuda()
    y[len(order):] = float("nan")                        # rows of no group
    y = y if f32 else y.to(torch.bfloat16)
    wts = rng.standard_normal((T, k)).astype(np.float32)
    wts[ids < 0] = np.nan                                # weights of choices that are none
    y64 = host(y)
    for w in (wts, None):
        out = zb.combine_rows(y, g, None if w is None else gpu(w))
        w64 = None if w is None else np.where(ids < 0, 0.0, w.astype(np.float64))
        want = grouped.combine(y64, place, w64)
        sizes = grouped.combine(np.abs(y64), place, None if w is None else np.abs(w64))
        assert (np.abs(host(out) - want) <= half_step(want) * (1 + 2.0 ** -10) + (k + 1) * 2.0 ** -24 * sizes + 1e-30).all()
        assert not out[0].any()
    # rows that lie apart, off any vector's boundary
    wide = torch.full((T, cols + 5), 7.0, dtype=torch.bfloat16, device="cuda")
    wide_y = torch.zeros(T * k, cols + 3, dtype=y.dtype, device="cuda")
    wide_y[:, 1:1 + cols] = y
    zb.combine_rows(wide_y[:, 1:1 + cols], g, gpu(wts), out=wide[:, 2:2 + cols])
    assert torch.equal(wide[:, 2:2 + cols], zb.combine_rows(y, g, gpu(wts)))
    wide[:, 2:2 + cols] = 7.0
    assert (wide == 7.0).all()


# ---- all of it --------------------------------------------------------------------------------------------------
def layer(E, H, I, seed, std=0.05):
    return [inputs.gaussian((I, H) if j < 2 else (H, I), std * (1 + 0.3 * ((e + j) % 3)), seed + 3 * e + j)
            for e in range(E) for j in range(3)]


def expected(ws, tok, ids, wts):
    """(out, bound) in float64.  h is rounded to bf16 once (half a step, through |w| |W2|), and may be on the other side of a
    step after fp32 sums (2e-6 of the magnitudes that they add); the output once more."""
    x = bf16_to_f64(tok)
    offsets, order, place = grouped.group(ids, len(ws) // 3)
    k = ids.shape[1]
    w1, w3, w2 = ([bf16_to_f64(w) for w in ws[j::3]] for j in range(3))
    g, u = grouped.products(x, order // k, offsets, w1), grouped.products(x, order // k, offsets, w3)
    h, ax = grouped.gated(g, u), np.abs(x)
    off = 2e-6 * (grouped.products(ax, order // k, offsets, [np.abs(w) for w in w1]) * 1.1 * np.abs(u) +
                  grouped.products(ax, order // k, offsets, [np.abs(w) for w in w3]) * np.abs(grouped.gated(g, 1.0)))
    here = np.arange(len(order))
    y = grouped.products(h, here, offsets, w2)
    slack = grouped.products(half_step(h) + np.abs(h) * 4e-6 + off, here, offsets, [np.abs(w) for w in w2])
    out = grouped.combine(y, place, wts)
    slack = grouped.combine(slack, place, None if wts is None else np.abs(wts))
    return out, half_step(out) + np.abs(out) * 1e-5 + slack + 1e-30


@pytest.mark.parametrize("T,E,k,H,I", [(1, 4, 2, 512, 768), (300, 9, 3, 264, 200), (1500, 4, 2, 256, 136), (700, 16, 8, 128, 64)])
def test_prompt_of_a_layer(zb, kernel, T, E, k, H, I):
    import torch
    ws = layer(E, H, I, 500 + E)
    ex = zb.ResidentExperts([gpu(w.view(np.int16)) for w in ws], H, I)
    tok = inputs.tokens(T, H, seed=T)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=T)
    if T > 1:
        ids[3] = -1
        ids[4, 0] = -1
        ids[5] = ids[5, 0]            # an expert listed k times counts with all its weights
    for w in (wts, None):
        out = ex.ffn_prompt(gpu(tok.view(np.int16)), gpu(ids), None if w is None else gpu(w))
        want, bound = expected(ws, tok, ids, w)
        got = bf16_to_f64(out.cpu().numpy().view(np.uint16))
        assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())
    assert int(ex.status.item()) == 0
    if T > 256:
        with pytest.raises(zb.ZipMoEError):
            ex.ffn(gpu(tok.view(np.int16)), gpu(ids), gpu(wts))
    ids[0, 0] = E
    ex.ffn_prompt(gpu(tok.view(np.int16)), gpu(ids), gpu(wts))
    assert int(ex.status.item()) == 1
    ex.status.zero_()
    assert ex.ffn_prompt(gpu(tok[:0].view(np.int16)), gpu(ids[:0]), gpu(wts[:0])).shape == (0, H)
    torch.cuda.synchronize()


def test_prompt_on_streams_and_in_a_graph(zb, kernel):
    """Two streams at once, and a captured prompt replayed on other inputs while eager calls run between the replays."""
    import torch
    T, E, k, H, I = 400, 6, 2, 256, 136
    ws = layer(E, H, I, 40)
    ex = zb.ResidentExperts([gpu(w.view(np.int16)) for w in ws], H, I)
    ins = []
    for seed in range(3):
        tok = inputs.tokens(T, H, seed=seed)
        ids, wts = inputs.routing(T, n_experts=E, k=k, seed=seed)
        ins.append((gpu(tok.view(np.int16)), gpu(ids), gpu(wts)))
    want = [ex.ffn_prompt(*i) for i in ins]
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    for _ in range(4):
        got = [ex.ffn_prompt(*i, stream=s) for i, s in zip(ins, streams)]
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    fixed = [t.clone() for t in ins[0]]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = ex.ffn_prompt(*fixed)
    for i, w in zip(ins, want):
        for a, b in zip(fixed, i):
            a.copy_(b)
        graph.replay()
        other = ex.ffn_prompt(*ins[1])
        torch.cuda.synchronize()
        assert torch.equal(out, w) and torch.equal(other, want[1])
    assert int(ex.status.item()) == 0


def test_first_prompt_within_a_capture(zb):
    """Evenly spaced experts need nothing on the device; others are described before."""
    import torch
    T, E, k, H, I = 300, 4, 2, 128, 72
    ws = layer(E, H, I, 90)
    tok, (ids, wts) = inputs.tokens(T, H, seed=1), inputs.routing(T, n_experts=E, k=k, seed=1)
    args = gpu(tok.view(np.int16)), gpu(ids), gpu(wts)
    flat = gpu(np.concatenate([w.ravel() for w in ws]).view(np.int16))
    even = zb.ResidentExperts(list(flat.view(3 * E, H * I)), H, I)
    apart = zb.ResidentExperts([gpu(w.view(np.int16)) for w in reversed(ws)][::-1], H, I)
    want = apart.ffn_prompt(*args)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = even.ffn_prompt(*args)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)
    fresh = zb.ResidentExperts([gpu(w.view(np.int16)) for w in reversed(ws)][::-1], H, I)
    if not fresh.struct.even:
        refused = []
        with torch.cuda.graph(torch.cuda.CUDAGraph()):
            args[0].add_(0)
            try:
                fresh.ffn_prompt(*args)
            except ValueError as err:
                refused.append(err)
        assert refused


def test_offsets_beyond_32_bits(zb, kernel):
    """Outputs, rows of x and sums that begin more than 2^32 bytes and elements into their buffers."""
    import torch
    R, N, K, pitch = 300000, 16384, 64, 16384
    x, w = coarse((R, K), 30, 1 / 16), coarse((2, N, K), 31, 1 / 64)
    wide = torch.empty(R, pitch, dtype=torch.bfloat16, device="cuda")
    wide[:, 512:512 + K] = bf16(x)
    ids = np.zeros((R, 1), np.int32)
    ids[R - 70:] = 1
    g = zb.group_tokens(gpu(ids), 2)
    m = zb.GroupedMatrix(list(bf16(w)))
    out = m.product(wide[:, 512:512 + K], g)
    rows = np.r_[0:3, R // 2:R // 2 + 3, R - 72:R]
    want = np.stack([x[r] @ w[ids[r, 0]].T for r in rows])
    assert torch.equal(out[gpu(rows)], torch.from_numpy(want).cuda().to(torch.bfloat16)) and int(m.status.item()) == 0
    del wide
    back = zb.combine_rows(out, g, None)
    assert torch.equal(back, out)


@pytest.mark.parametrize("T", [5, 700])
def test_a_wait_that_runs_out_is_reported(zb, kernel, T):
    """The weights' barriers armed for more than their copies bring: the call ends and says so, and the next one is sound."""
    import torch
    E, K, N = 4, 512, 300
    x, w = coarse((T, K), 16, 1 / 16), coarse((E, N, K), 17, 1 / 64)
    ids = routing(T, 1, E, 18)
    g = zb.group_tokens(gpu(ids), E)
    m = zb.GroupedMatrix(list(bf16(w)))
    want = m.product(bf16(x), g, gather=True)
    torch.cuda.synchronize()
    zb.zipmoe_test_wait_fault(16, 1)
    try:
        m.product(bf16(x), g, gather=True)
        torch.cuda.synchronize()
    finally:
        zb.zipmoe_test_wait_fault(0, 0)
    assert int(m.status.item()) == 3
    m.status.zero_()
    assert torch.equal(m.product(bf16(x), g, gather=True), want) and int(m.status.item()) == 0


def test_refusals_of_the_classes(zb):
    import torch
    E, K, N, T = 3, 64, 40, 6
    w = [torch.zeros(N, K, dtype=torch.bfloat16, device="cuda") for _ in range(E)]
    q = [torch.zeros(N, K, dtype=torch.int8, device="cuda") for _ in range(E)]
    s = torch.ones(E, N, device="cuda")
    x = torch.zeros(T, K, dtype=torch.bfloat16, device="cuda")
    g = zb.group_tokens(torch.zeros(T, 1, dtype=torch.int32, device="cuda"), E)
    for bad in (lambda: zb.GroupedMatrix([]), lambda: zb.GroupedMatrix(w, up=w[:2]), lambda: zb.GroupedMatrix(w, scales=s),
                lambda: zb.GroupedMatrix(q), lambda: zb.GroupedMatrix(q, up=q, scales=s), lambda: zb.GroupedMatrix(w[:2] + [q[0]]),
                lambda: zb.GroupedMatrix(w[:2] + [w[0].t()]), lambda: zb.GroupedMatrix([w[0].cpu()]),
                lambda: zb.GroupedMatrix(q, scales=s[:2]), lambda: zb.GroupedMatrix(w).product(x), lambda: zb.GroupedMatrix(w).product(x[:5], g),
                lambda: zb.GroupedMatrix(w).product(x.float(), g), lambda: zb.GroupedMatrix(w).product(x, g, row_scales=s),
                lambda: zb.GroupedMatrix(w[:2]).product(x, g), lambda: zb.GroupedMatrix(w[:1]).product(x, gather=True),
                lambda: zb.GroupedMatrix(q, scales=s).product(torch.zeros(T, K, dtype=torch.int8, device="cuda"), g),
                lambda: zb.GroupedMatrix(w).product(x, g, out=torch.zeros(T, N + 1, dtype=torch.bfloat16, device="cuda")),
                lambda: zb.GroupedMatrix(w).product(x.t().contiguous().t(), g), lambda: zb.group_tokens(torch.zeros(3, 2, device="cuda"), 4),
                lambda: zb.group_tokens(torch.zeros(3, 2, dtype=torch.int32), 4), lambda: zb.combine_rows(torch.zeros(5, 8, device="cuda"), g, None),
                lambda: zb.combine_rows(torch.zeros(T, 8, device="cuda"), g, torch.zeros(T, 2, device="cuda")),
                lambda: zb.quantize_rows(torch.zeros(3, 8, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(zb.ZipMoEError):
        zb.GroupedMatrix([torch.zeros(8, 12, dtype=torch.bfloat16, device="cuda")])
    with pytest.raises(zb.ZipMoEError):       # rows of x that no 16-byte copy can start at
        zb.GroupedMatrix(w).product(torch.zeros(T, K + 4, dtype=torch.bfloat16, device="cuda")[:, :K], g)
