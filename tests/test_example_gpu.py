"""The example's sublayer - norm, router, recovered and compressed experts together - against the fp64 oracles."""
import importlib.util
import os

import numpy as np
import pytest

from oracle import sublayer
from oracle.ffn import bf16_to_f64, silu
from paper_2601_21198_b200 import build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def example():
    build.build()
    spec = importlib.util.spec_from_file_location("expert_sublayer", os.path.join(ROOT, "examples", "expert_sublayer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def bits(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("resident", [0, 3, 6])
@pytest.mark.parametrize("T", [1, 13])
def test_sublayer_against_the_oracles(example, T, resident):
    import torch
    E, H, I, k = 6, 512, 768, 2
    ws, layer = example.build(E, resident, H, I, k, seed=resident)
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    residual = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    x64, r64 = bf16_to_f64(bits(x)), bf16_to_f64(bits(residual))
    y, q, scales = layer.forward(x, residual)
    # norm: the residual in place, the 8-bit rows
    h64, n64 = sublayer.add_rmsnorm(x64, r64, bf16_to_f64(bits(layer.norm.weight)), 1e-6)
    assert (np.abs(bf16_to_f64(bits(residual)) - h64) <= np.abs(h64) * 2.0 ** -8).all()
    s = scales.cpu().numpy().astype(np.float64)
    assert (np.abs(sublayer.e4m3_to_f64(q.view(torch.uint8).cpu().numpy()) * s - n64) <= np.maximum(np.abs(n64) * 2.0 ** -4, s * 2.0 ** -10) * 1.01).all()
    # router and experts, from the rows that they were given
    h = torch.empty_like(x)
    layer.norm.add_norm(x, torch.from_numpy((r64).astype(np.float32)).cuda().to(torch.bfloat16), out=h)
    rows = bf16_to_f64(bits(h))
    logits = rows @ bf16_to_f64(bits(layer.router.gate)).T
    ids = sublayer.choose(logits, k)
    w = sublayer.weights_of(logits, ids)
    want = np.zeros((T, H))
    for t in range(T):
        for j in range(k):
            w1, w3, w2 = (bf16_to_f64(ws[3 * ids[t, j] + i]) for i in range(3))
            want[t] += w[t, j] * (w2 @ (silu(w1 @ rows[t]) * (w3 @ rows[t])))
    got = bf16_to_f64(bits(y))
    assert np.linalg.norm(got - want) <= 1e-2 * np.linalg.norm(want)


def test_command_runs(example, capsys):
    example.main(["--tokens", "2", "--experts", "4", "--resident", "2", "--hidden", "512", "--inter", "512"])
    assert "us per sublayer" in capsys.readouterr().out
