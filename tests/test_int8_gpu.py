"""Rows in 8-bit integers and the dense product of them on the GPU against the fp64 oracle.

127 x is exact in fp32 and 127 x / a is either half way between two integers or at least 1 / (2 * 255 * 127) of its value away
from there, so the integers have to be the oracle's; the scale is one fp32 division.  A product's integers are exact, its
conversion to fp32 and the two scales are three roundings (3 * 2^-24), the output is rounded to bf16 once (2^-8)."""
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


def gpu(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def half_step(v):
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - 8)


@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 16), (3, 7), (5, 2048), (4, 2056), (9, 4096), (2, 8200), (3, 14336), (2, 16640), (1, 32768), (2, 40000),
                                       (1, 65536), (300, 1408), (1000, 100), (2, 65535)])
def test_rows(zb, rows, cols):
    import torch
    x = inputs.tokens(rows, cols, seed=cols)
    x[0, 0] = 0xBF80 if cols > 1 else x[0, 0]         # -1
    if rows > 2:
        x[1] = 0                                      # a row of zeros
        x[2] = x[2] & 0x80FF | 0x3F80                 # values in [1, 2): many of them half way between two integers
    q, s = zb.quantize_rows(gpu(x.view(np.int16)))
    want, scales = grouped.quantize(bf16_to_f64(x))
    assert np.array_equal(q.cpu().numpy(), want)
    assert np.array_equal(s.cpu().numpy(), (np.abs(bf16_to_f64(x)).max(axis=1).astype(np.float32) / np.float32(127)))
    assert np.allclose(s.cpu().numpy(), scales, rtol=2.0 ** -23)
    # rows that lie apart and start anywhere
    wide = torch.full((rows, cols + 9), float("nan"), dtype=torch.bfloat16, device="cuda").view(torch.int16)
    wide[:, 1:1 + cols] = gpu(x.view(np.int16))
    out = torch.full((rows, cols + 5), 77, dtype=torch.int8, device="cuda")
    zb.quantize_rows(wide[:, 1:1 + cols], q=out[:, 3:3 + cols])
    assert torch.equal(out[:, 3:3 + cols], q)
    out[:, 3:3 + cols] = 77
    assert (out == 77).all()


def test_every_pattern_against_every_mantissa(zb):
    """All finite bf16 patterns of magnitude at most a, for every mantissa of a, in two binades and at both ends."""
    import torch
    every = np.arange(65536, dtype=np.uint16)
    mag = every & 0x7FFF
    rows = [np.where(mag <= top, every, 0) for m in range(128) for top in (0x3F80 + m, 0x0080 + m)] + [np.where(mag <= 0x7F7F, every, 0)]
    x = np.stack(rows).astype(np.uint16)
    q, s = zb.quantize_rows(gpu(x.view(np.int16)))
    want, _ = grouped.quantize(bf16_to_f64(x))
    assert np.array_equal(q.cpu().numpy(), want)
    assert torch.isfinite(s).all()


def test_rows_that_are_not_finite(zb):
    import torch
    x = torch.ones(5, 64, dtype=torch.bfloat16, device="cuda")
    x[1, 3], x[2, 60], x[3, 0] = float("nan"), float("inf"), float("-inf")
    q, s = zb.quantize_rows(x)
    assert s.isnan().tolist() == [False, True, True, True, False] and not q[1:4].any() and (q[0] == 127).all()
    lin = zb.Int8Linear(torch.ones(40, 64, dtype=torch.int8, device="cuda"), torch.ones(40, device="cuda"))
    out = lin.product(x)
    assert out[1:4].isnan().all() and (out[0] == 64).all() and (out[4] == 64).all()
    assert zb.quantize_rows(x[:0])[0].shape == (0, 64)


@pytest.mark.parametrize("T,K,N", [(1, 16, 1), (1, 4096, 300), (3, 48, 7), (16, 1424, 129), (17, 2048, 64), (64, 256, 2051), (65, 272, 130), (300, 1040, 257),
                                   (513, 128, 520), (1531, 1424, 130), (5, 16384, 40), (1, 65536, 24), (300, 65536, 24)])
def test_linear(zb, kernel, T, K, N):
    import torch
    rng = np.random.default_rng(K)
    x = inputs.tokens(T, K, seed=T)
    w, s = rng.integers(-128, 128, (N, K), dtype=np.int8), (rng.random(N) * 1e-3 + 1e-4).astype(np.float32)
    lin = zb.Int8Linear(gpu(w), gpu(s))
    out = torch.empty(T, N, device="cuda")
    lin.product(gpu(x.view(np.int16)), out=out)
    q, _ = grouped.quantize(bf16_to_f64(x))
    scales = np.abs(bf16_to_f64(x)).max(axis=1).astype(np.float32) / np.float32(127)
    acc = q.astype(np.float64) @ w.astype(np.float64).T                        # whole numbers below 2^53: exact
    want = (acc.astype(np.float32) * scales[:, None]).astype(np.float32) * s
    assert np.array_equal(out.cpu().numpy(), want)
    exact = acc * (np.abs(bf16_to_f64(x)).max(axis=1) / 127)[:, None] * s.astype(np.float64)
    half = lin.product(gpu(x.view(np.int16)).view(torch.bfloat16))
    assert half.dtype == torch.bfloat16
    # (the scale's own rounding is the fourth)
    assert (np.abs(half.double().cpu().numpy() - exact) <= half_step(exact) * (1 + 2.0 ** -10) + 4 * 2.0 ** -24 * np.abs(exact)).all()
    assert int(lin.status.item()) == 0


def test_largest_sums(zb, kernel):
    """The longest rows of the largest integers: 65536 * 128 * 128 = 2^30."""
    import torch
    K, N = 65536, 16
    w = torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    m = zb.GroupedMatrix([w], scales=torch.ones(N, device="cuda"))
    out = torch.empty(3, N, device="cuda")
    for v, want in ((-128, 2.0 ** 30), (127, -127.0 * 2 ** 23)):
        m.product(torch.full((3, K), v, dtype=torch.int8, device="cuda"), row_scales=torch.ones(3, device="cuda"), out=out)
        assert (out == want).all()


def test_weights_from_bf16_graph_and_stream(zb):
    import torch
    T, K, N = 70, 512, 200
    weight = inputs.gaussian((N, K), 0.02, 3)
    lin = zb.Int8Linear.from_bf16(gpu(weight.view(np.int16)))
    qw, sw = grouped.quantize(bf16_to_f64(weight))
    x = gpu(inputs.tokens(T, K, seed=1).view(np.int16)).view(torch.bfloat16)

    def check(out, x):
        qx, sx = grouped.quantize(x.double().cpu().numpy())
        want = (qx @ qw.T) * sx[:, None] * sw
        assert (np.abs(out.double().cpu().numpy() - want) <= half_step(want) * (1 + 2.0 ** -10) + 8 * 2.0 ** -24 * np.abs(want)).all()

    check(lin.product(x), x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out = lin.product(x, stream=side)
    side.synchronize()
    check(out, x)
    fixed = x.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = lin.product(fixed)
    other = gpu(inputs.tokens(T, K, seed=2).view(np.int16)).view(torch.bfloat16)
    fixed.copy_(other)
    graph.replay()
    torch.cuda.synchronize()
    check(out, other)
