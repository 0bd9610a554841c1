"""Forms of the grouped products that other tests leave out: pairs of bf16 with fp32 rows, and 8-bit weights in no order with rows
that lie apart.

Operands on coarse grids make the two sums of a pair exact.  The gated activation adds the fp32 exponential (2 units of 2^-23,
and |g| of them from its argument), a division and two products: (8 + 2 |g|) * 2^-23 of the value.  8-bit sums are exact, and
each of their two scales is one fp32 product."""
import numpy as np
import pytest

from oracle import grouped
from paper_2601_21198_b200 import build

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


def coarse(shape, seed, step):
    """Whole multiples of `step`, at most 8 of them: products of two such and sums of 2^17 of those are exact in fp32."""
    rng = np.random.default_rng(seed)
    return np.clip(np.rint(rng.standard_normal(shape) * 2.5), -8, 8) * step


def gpu(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def bf16(a):
    import torch
    return gpu(np.asarray(a, np.float32)).to(torch.bfloat16)


def routing(T, k, E, seed):
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(E)[:k] for _ in range(T)]).astype(np.int32)
    if T > 4:
        ids[rng.random((T, k)) < 0.1] = -1
    return ids


def check_gated(out, first, second):
    want = grouped.gated(first, second)
    bound = np.abs(want) * (8 + 2 * np.abs(first)) * 2.0 ** -23 + 1e-30
    assert (np.abs(out.double().cpu().numpy() - want) <= bound).all()


@pytest.mark.parametrize("T,E,k,K,N", [(1, 1, 1, 8, 8), (5, 3, 2, 72, 40), (65, 4, 1, 256, 129), (300, 2, 1, 192, 384), (777, 60, 4, 264, 136),
                                       (1100, 3, 2, 1032, 520), (513, 1, 1, 512, 768)])
@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("apart", [0, 3])
def test_pairs_with_rows_of_fp32(zb, kernel, T, E, k, K, N, gather, apart):
    """apart: elements between rows of the output; three of them put most rows off any vector's boundary."""
    import torch
    ids = routing(T, k, E, T)
    g = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    x, w1, w3 = coarse((T if gather else T * k, K), 3, 1 / 16), coarse((E, N, K), 4, 1 / 64), coarse((E, N, K), 5, 1 / 64)
    m = zb.GroupedMatrix(list(bf16(w1)), up=list(bf16(w3)))
    src = order // k if gather else np.arange(len(order))
    wide = torch.full((T * k, N + apart), 7.0, device="cuda")
    m.product(bf16(x), g, gather=gather, out=wide[:, apart:])
    check_gated(wide[:len(order), apart:], grouped.products(x, src, offsets, w1), grouped.products(x, src, offsets, w3))
    wide[:len(order), apart:] = 7.0
    assert (wide == 7.0).all() and int(m.status.item()) == 0


@pytest.mark.parametrize("T,K,N", [(6, 144, 90), (500, 272, 300)])
@pytest.mark.parametrize("pair", [False, True])
@pytest.mark.parametrize("gather", [False, True])
def test_8_bits_scattered_and_apart(zb, kernel, T, K, N, pair, gather):
    """Weights each in an allocation of its own, in no order; rows of x 48 bytes apart, between other values."""
    import torch
    E, k, rng = 5, 2, np.random.default_rng(K)
    ids = routing(T, k, E, 9)
    g = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    rows, src = (T, order // k) if gather else (T * k, np.arange(len(order)))
    x, w = rng.integers(-128, 128, (rows, K), dtype=np.int8), rng.integers(-128, 128, (2, E, N, K), dtype=np.int8)
    sx, sw = (rng.random(rows) / 64 + 1e-3).astype(np.float32), (rng.random((2, E, N)) / 64 + 1e-3).astype(np.float32)
    pool = torch.empty(2 * E, N * K + 4096, dtype=torch.int8, device="cuda")
    apart = [[None] * E, [None] * E]
    for place, (j, e) in enumerate(rng.permutation([(j, e) for j in range(2) for e in range(E)])):
        apart[j][e] = pool[place, 16 * place:16 * place + N * K].view(N, K).copy_(gpu(w[j, e]))
    m = zb.GroupedMatrix(apart[0], up=apart[1] if pair else None, scales=gpu(sw[0]), up_scales=gpu(sw[1]) if pair else None)
    assert not m.struct.even
    wide = torch.full((rows, K + 48), 99, dtype=torch.int8, device="cuda")
    wide[:, 16:16 + K] = gpu(x)
    out = torch.full((T * k, N), 7.0, device="cuda")
    m.product(wide[:, 16:16 + K], g, gather=gather, row_scales=gpu(sx), out=out)
    of = np.repeat(np.arange(E), np.diff(offsets))
    scaled = [(grouped.products(x.astype(np.float64), src, offsets, w[j].astype(np.float64)).astype(np.float32) * sx[src][:, None]) * sw[j][of]
              for j in range(2)]
    if pair:
        check_gated(out[:len(order)], *[s.astype(np.float64) for s in scaled])
    else:
        assert np.array_equal(out[:len(order)].cpu().numpy(), scaled[0])
    assert (out[len(order):] == 7.0).all() and int(m.status.item()) == 0
