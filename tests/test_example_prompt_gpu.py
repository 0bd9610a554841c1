"""The example's sublayer on a prompt of more tokens than one call on recovered experts takes: its experts run as grouped
products there.  Against the fp64 formula with the router's own choice; h between the products is bf16 (2^-9 of each of a sum
of independent roundings) and so is the output, so the whole is within 1e-2 of its norm as the shorter calls are."""
import importlib.util
import os

import numpy as np
import pytest

from oracle.ffn import bf16_to_f64, silu
from paper_2601_21198_b200 import build

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def bits(t):
    import torch
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("resident", [2, 4])
def test_prompt(resident):
    import torch
    build.build()
    spec = importlib.util.spec_from_file_location("expert_sublayer", os.path.join(ROOT, "examples", "expert_sublayer.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    T, E, H, I, k = 300, 4, 256, 512, 2
    ws, layer = example.build(E, resident, H, I, k, seed=3)
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    residual = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    h = layer.norm.add_norm(x, residual.clone())
    ids, weights = layer.router.route(h)
    y, _, _ = layer.forward(x, residual)
    torch.cuda.synchronize()
    assert int(layer.recovered.status.item()) == 0
    rows, ids, weights = bf16_to_f64(bits(h)), ids.cpu().numpy(), weights.cpu().numpy().astype(np.float64)
    want = np.zeros((T, H))
    for e in range(E):
        w1, w3, w2 = (bf16_to_f64(ws[3 * e + i]) for i in range(3))
        t, j = np.nonzero(ids == e)
        np.add.at(want, t, weights[t, j][:, None] * ((silu(rows[t] @ w1.T) * (rows[t] @ w3.T)) @ w2.T))
    assert np.linalg.norm(bf16_to_f64(bits(y)) - want) <= 1e-2 * np.linalg.norm(want)
