"""The example's layer with some experts recovered and the others compressed: an expert touches only the tokens that chose
it, and any number of experts may stay compressed."""
import importlib.util
import os

import numpy as np
import pytest

from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
E, H, I, K = 6, 512, 768, 2


@pytest.fixture(scope="module")
def example():
    build.build()
    spec = importlib.util.spec_from_file_location("expert_sublayer", os.path.join(ROOT, "examples", "expert_sublayer.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def weights():
    return [inputs.gaussian((I, H) if j % 3 < 2 else (H, I), 0.02, 40 + j) for j in range(3 * E)]


def layer_of(example, ws, resident):
    import torch
    from paper_2601_21198_b200 import binding as zb
    blobs = [zb.zipmoe_encode(w, layout=zb.LAYOUT_BLOCKED, chunk_elems=65536) for w in ws]
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    gate = (0.05 * torch.randn(len(ws) // 3, H, generator=g, device="cuda")).to(torch.bfloat16)
    return example.ExpertSublayer(torch.ones(H, dtype=torch.bfloat16, device="cuda"), gate, K, blobs, H, I, resident)


def forward(layer, T):
    """The output, and which experts every token chose."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    h = layer.norm.add_norm(x, torch.zeros_like(x))
    ids, _ = layer.router.route(h)
    return layer.forward(x, torch.zeros_like(x))[0], ids.cpu().numpy()


@pytest.mark.parametrize("T", [1, 13, 40])
@pytest.mark.parametrize("poisoned", [3, 4, 5])
def test_an_infinite_expert_touches_only_its_own_tokens(example, T, poisoned):
    sound, _ = forward(layer_of(example, weights(), 3), T)
    ws = weights()
    ws[3 * poisoned + 2][:, 5] = 0x7F80                # +inf in every row of w2
    got, ids = forward(layer_of(example, ws, 3), T)
    has = (ids == poisoned).any(axis=1)
    got, sound = got.float().cpu().numpy(), sound.float().cpu().numpy()
    assert np.array_equal(got[~has], sound[~has]) and np.isfinite(sound).all()
    assert not np.isfinite(got[has]).any()


@pytest.mark.parametrize("resident", [1, 5])
@pytest.mark.parametrize("T", [1, 40])
def test_any_number_of_experts_may_stay_compressed(example, T, resident):
    ws = weights()
    want, _ = forward(layer_of(example, ws, E), T)
    got, _ = forward(layer_of(example, ws, resident), T)
    got, want = got.float().cpu().numpy(), want.float().cpu().numpy()
    # the last rounding to bf16 of either side, that of a compressed expert's result before it is weighed, and the h that the
    # two calls' sums round to different sides: half a step each, 2^-8 of a value
    assert np.linalg.norm(got - want) <= 4 * 2.0 ** -8 * np.linalg.norm(want)
