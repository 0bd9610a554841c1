"""Weights that are described while their stream has work left, and used on another stream at once: no wait of the caller's stands
between the two, so what the constructors put on the device has to be there when they return."""
import numpy as np
import pytest

from oracle import grouped
from oracle.ffn import bf16_to_f64
from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu
BUSY = 200_000_000      # clock cycles, 0.1 s


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def gpu(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def test_rounded_weights_on_another_stream(zb):
    import torch
    T, K, N = 40, 512, 264
    weight, tokens = inputs.gaussian((N, K), 0.02, 3), inputs.tokens(T, K, seed=1)
    w, x, side = gpu(weight.view(np.int16)), gpu(tokens.view(np.int16)), torch.cuda.Stream()
    want = zb.Int8Linear.from_bf16(w).product(x)
    (qx, sx), (qw, sw) = grouped.quantize(bf16_to_f64(tokens)), grouped.quantize(bf16_to_f64(weight))
    exact = (qx @ qw.T) * sx[:, None] * sw
    assert np.allclose(bf16_to_f64(want.cpu().numpy().view(np.uint16)), exact, rtol=2.0 ** -8 * 1.01, atol=1e-30)
    for _ in range(3):
        torch.empty(N, K, dtype=torch.int8, device="cuda").fill_(77)      # what the pool gives out next is no zeros
        torch.cuda.synchronize()
        torch.cuda._sleep(BUSY)
        linear = zb.Int8Linear.from_bf16(w)
        got = linear.product(x, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(got, want) and int(linear.status.item()) == 0


@pytest.mark.parametrize("int8", [False, True])
def test_an_error_on_another_stream_is_not_cleared(zb, int8):
    """The status word is zeroed before the constructor returns, not after the first call has set it."""
    import torch
    rows, K, N, side = 6, 64, 40, torch.cuda.Stream()
    kind = torch.int8 if int8 else torch.bfloat16
    w, x = torch.zeros(2, N, K, dtype=kind, device="cuda"), torch.zeros(rows, K, dtype=kind, device="cuda")
    scales = dict(scales=torch.ones(2, N, device="cuda")) if int8 else {}
    row_scales = torch.ones(rows, device="cuda") if int8 else None
    wrong = gpu(np.array([0, 4, 3], np.int32)), gpu(np.arange(rows, dtype=np.int32)), gpu(np.zeros((rows, 1), np.int32))
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    m = zb.GroupedMatrix(list(w), **scales)
    m.product(x, zb.TokenGroups(*wrong, 2), row_scales=row_scales, stream=side)
    torch.cuda.synchronize()
    assert int(m.status.item()) == 1
