"""8-bit products whose scales are subnormal numbers, or whose scaled sums are: rows of tiny numbers, weights that make them
ordinary again.  The sum is exact and each of the two scales one fp32 product, so the result is that of the same two products on
the CPU, bit for bit, and in bf16 the nearest to it."""
import numpy as np
import pytest

from oracle import grouped
from oracle.ffn import bf16_to_f64
from paper_2601_21198_b200 import build

pytestmark = pytest.mark.gpu
TOPS = [2.0 ** -133, 2.0 ** -130 * 1.5, 2.0 ** -126, 2.0 ** -120 * 1.25, 2.0 ** -119, 2.0 ** -100, 1.0]      # of a row: its largest magnitude


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


def column_scales(rng, shape):
    return (rng.random(shape) + 0.5).astype(np.float32) * np.float32(2.0) ** rng.integers(-140, 90, shape).astype(np.float32)


def same(out, want):
    import torch
    assert torch.equal(out.cpu(), torch.from_numpy(want).to(out.dtype))


@pytest.mark.parametrize("T,K,N", [(7, 256, 130), (300, 144, 520)])
def test_linear_of_tiny_rows(zb, kernel, T, K, N):
    import torch
    rng = np.random.default_rng(T)
    top = np.array(TOPS)[np.arange(T) % len(TOPS)]
    x = torch.from_numpy((rng.uniform(-1, 1, (T, K)) * top[:, None])).to(torch.bfloat16)
    x[:, 0] = torch.from_numpy(top).to(torch.bfloat16)
    bits = x.view(torch.int16)
    values = bf16_to_f64(bits.numpy().view(np.uint16))
    w, s = rng.integers(-127, 128, (N, K), dtype=np.int8), column_scales(rng, N)
    q, _ = grouped.quantize(values)
    scales = np.abs(values).max(axis=1).astype(np.float32) / np.float32(127)
    assert (scales > 0).all() and (scales < 2.0 ** -126).any()
    with np.errstate(all="ignore"):
        want = ((q @ w.astype(np.int64).T).astype(np.float32) * scales[:, None]).astype(np.float32) * s
    linear = zb.Int8Linear(gpu(w), gpu(s))
    out = torch.empty(T, N, device="cuda")
    same(linear.product(bits.cuda(), out=out), want)
    same(linear.product(x.cuda()), want)


@pytest.mark.parametrize("T", [9, 500])
@pytest.mark.parametrize("gather", [False, True])
def test_groups_of_tiny_rows(zb, kernel, T, gather):
    import torch
    E, k, K, N = 3, 2, 160, 72
    rng = np.random.default_rng(T)
    ids = rng.integers(0, E, (T, k)).astype(np.int32)
    groups = zb.group_tokens(gpu(ids), E)
    offsets, order, _ = grouped.group(ids, E)
    rows, src = (T, order // k) if gather else (T * k, np.arange(T * k))
    x, w = rng.integers(-128, 128, (rows, K), dtype=np.int8), rng.integers(-128, 128, (E, N, K), dtype=np.int8)
    sx, sw = (np.array(TOPS)[np.arange(rows) % len(TOPS)] / 127).astype(np.float32), column_scales(rng, (E, N))
    acc = grouped.products(x.astype(np.float64), src, offsets, w.astype(np.float64))
    with np.errstate(all="ignore"):
        want = (acc.astype(np.float32) * sx[src][:, None]).astype(np.float32) * sw[np.repeat(np.arange(E), np.diff(offsets))]
    m = zb.GroupedMatrix(list(gpu(w)), scales=gpu(sw))
    for dtype in (torch.float32, torch.bfloat16):
        out = torch.empty(T * k, N, dtype=dtype, device="cuda")
        same(m.product(gpu(x), groups, gather=gather, row_scales=gpu(sx), out=out), want)
