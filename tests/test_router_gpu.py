"""zipmoe_route on the GPU against the fp64 oracle.  The choice is compared exactly on data whose logits are exact in
fp32 whatever the order of the sums (activations and gate on coarse grids); the logits on arbitrary data within the
worst-case bound of an fp32 sum, hidden * 2^-24 * sum |x g|; the weights against the softmax of the call's own logits
(exp and division of fp32: a few units of 2^-23, and |logit - top| of them for the reduction of the argument)."""
import numpy as np
import pytest

from oracle import sublayer
from oracle.ffn import bf16_to_f64
from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def exact_data(T, H, E, seed, levels=16):
    """x and gate as float64 whose products sum without rounding in fp32."""
    rng = np.random.default_rng(seed)
    x = np.clip(np.rint(rng.standard_normal((T, H)) * levels), -100, 100) / levels
    g = np.clip(np.rint(rng.standard_normal((E, H)) * 20), -100, 100) / 1024
    return x, g


def to_bf16(a):
    import torch
    return torch.from_numpy(np.asarray(a, np.float32)).cuda().to(torch.bfloat16)


def check_weights(w, logits, ids, renormalise):
    want = sublayer.weights_of(logits, ids, renormalise)
    finite = np.where(np.isfinite(logits), logits, 0.0)
    spread = np.abs(logits.max(axis=1, keepdims=True) - np.take_along_axis(finite, np.maximum(ids, 0).astype(np.int64), 1))
    spread = np.where(ids >= 0, spread, 0.0)
    assert (np.abs(w - want) <= want * (16 + 2 * spread) * 2.0 ** -23 + 1e-37).all()
    assert not w[ids < 0].any()


@pytest.mark.parametrize("T,H,E,k", [(1, 2048, 64, 6), (1, 8, 1, 1), (2, 64, 3, 2), (5, 4096, 8, 2), (17, 1416, 60, 4),
                                     (33, 2048, 256, 8), (127, 512, 128, 1), (128, 256, 31, 8), (129, 72, 33, 5), (300, 1024, 64, 6),
                                     (1000, 2056, 96, 3), (64, 4096, 255, 8), (3, 32768, 16, 2)])
@pytest.mark.parametrize("renormalise", [True, False])
def test_choice_and_weights(zb, T, H, E, k, renormalise):
    import torch
    x, g = exact_data(T, H, E, T + H + E)
    rng = np.random.default_rng(E)
    b = np.rint(rng.standard_normal(E) * 4096) / 16384
    logits = torch.empty(T, E, device="cuda")
    router = zb.Router(to_bf16(g), k, bias=torch.from_numpy(b.astype(np.float32)).cuda(), renormalise=renormalise)
    ids, w = router.route(to_bf16(x), logits=logits)
    want = x @ g.T + b
    assert np.array_equal(logits.cpu().numpy().astype(np.float64), want)
    assert np.array_equal(ids.cpu().numpy(), sublayer.choose(want, k))
    check_weights(w.cpu().numpy().astype(np.float64), want, ids.cpu().numpy(), renormalise)
    assert int(router.status.item()) == 0
    # the same choice without the logits being asked for, and without a bias the unbiased one
    ids2, w2 = router.route(to_bf16(x))
    assert torch.equal(ids, ids2) and torch.equal(w, w2)
    ids3, _ = zb.Router(to_bf16(g), k).route(to_bf16(x))
    assert np.array_equal(ids3.cpu().numpy(), sublayer.choose(x @ g.T, k))


def test_logits_of_arbitrary_data(zb):
    import torch
    for T, H, E in ((3, 2048, 64), (200, 4096, 60), (64, 136, 256)):
        tok = inputs.tokens(T, H, seed=T)
        gate = inputs.gaussian((E, H), 0.02, 77 + E)
        logits = torch.empty(T, E, device="cuda")
        router = zb.Router(torch.from_numpy(gate.view(np.int16)).cuda(), 2)
        ids, w = router.route(torch.from_numpy(tok.view(np.int16)).cuda(), logits=logits)
        x, g = bf16_to_f64(tok), bf16_to_f64(gate)
        got = logits.cpu().numpy().astype(np.float64)
        assert (np.abs(got - x @ g.T) <= H * 2.0 ** -24 * (np.abs(x) @ np.abs(g).T)).all()
        assert np.array_equal(ids.cpu().numpy(), sublayer.choose(got, 2))
        check_weights(w.cpu().numpy().astype(np.float64), got, ids.cpu().numpy(), True)


def test_ties_take_the_lowest_index(zb):
    import torch
    E, k, H = 96, 6, 64
    g = np.zeros((E, H))
    g[40:] = g[:56] = 0.0
    ids, w = zb.Router(to_bf16(g), k).route(to_bf16(np.ones((9, H))))
    assert np.array_equal(ids.cpu().numpy(), np.tile(np.arange(k), (9, 1)))
    assert np.allclose(w.cpu().numpy(), 1 / k, rtol=1e-6)
    g[70] = g[33] = g[95] = 1.0 / 64
    g[3] = -1.0 / 64
    ids, _ = zb.Router(to_bf16(g), k).route(to_bf16(np.ones((9, H))))
    assert np.array_equal(ids.cpu().numpy(), np.tile([33, 70, 95, 0, 1, 2], (9, 1)))
    del torch


@pytest.mark.parametrize("renormalise", [True, False])
@pytest.mark.parametrize("E,left", [(64, 3), (64, 0), (5, 1), (256, 8), (40, 39)])
def test_experts_switched_off(zb, E, left, renormalise):
    """A bias of -inf: fewer than k experts, or none, are left."""
    import torch
    T, H, k = 20, 128, 5
    x, g = exact_data(T, H, E, 5)
    rng = np.random.default_rng(left)
    on = rng.permutation(E)[:left]
    b = np.full(E, -np.inf)
    b[on] = 0.25
    router = zb.Router(to_bf16(g), k, bias=torch.from_numpy(b.astype(np.float32)).cuda(), renormalise=renormalise)
    logits = torch.empty(T, E, device="cuda")
    ids, w = router.route(to_bf16(x), logits=logits)
    want = x @ g.T + b
    assert np.array_equal(logits.cpu().numpy().astype(np.float64), want)
    assert np.array_equal(ids.cpu().numpy(), sublayer.choose(want, k))
    assert (ids.cpu().numpy() >= 0).sum(axis=1).tolist() == [min(left, k)] * T
    w = w.cpu().numpy()
    if left == 0:
        assert not w.any()
    else:
        check_weights(w.astype(np.float64), want, ids.cpu().numpy(), renormalise)


def test_nan_and_infinite_logits(zb):
    import torch
    T, H, E, k = 5, 64, 32, 3
    x, g = exact_data(T, H, E, 8)
    x[1, 0] = np.nan
    b = np.zeros(E)
    tok = to_bf16(x)
    ids, w = zb.Router(to_bf16(g), k, bias=torch.from_numpy(b.astype(np.float32)).cuda()).route(tok)
    ids, w = ids.cpu().numpy(), w.cpu().numpy()
    assert ids[1].tolist() == [0, 1, 2] and np.isnan(w[1]).all()          # every logit is NaN: lowest indices, loud weights
    rest = [0, 2, 3, 4]
    assert np.array_equal(ids[rest], sublayer.choose((x @ g.T)[rest], k)) and np.isfinite(w[rest]).all()
    b[7], b[9] = np.nan, np.inf
    ids, w = zb.Router(to_bf16(g), k, bias=torch.from_numpy(b.astype(np.float32)).cuda()).route(tok)
    ids, w = ids.cpu().numpy(), w.cpu().numpy()
    assert (ids[rest, :2] == [7, 9]).all() and np.isnan(w).any(axis=1).all()


def test_wide_rows_no_tokens_and_another_stream(zb):
    import torch
    T, H, E, k = 70, 256, 24, 2
    x, g = exact_data(T, H, E, 3)
    router = zb.Router(to_bf16(g), k)
    wide = torch.full((T, 304), float("nan"), dtype=torch.bfloat16, device="cuda")
    wide[:, 16:16 + H] = to_bf16(x)
    want = sublayer.choose(x @ g.T, k)
    ids, _ = router.route(wide[:, 16:16 + H])
    assert np.array_equal(ids.cpu().numpy(), want)
    assert router.route(wide[:0, :H])[0].shape == (0, k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ids, _ = router.route(wide[:, 16:16 + H], stream=side)
    side.synchronize()
    assert np.array_equal(ids.cpu().numpy(), want)


def test_captured_into_a_graph(zb):
    import torch
    T, H, E, k = 9, 512, 64, 6
    x, g = exact_data(T, H, E, 21)
    router = zb.Router(to_bf16(g), k)
    tok = to_bf16(x)
    ids, w = router.route(tok)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        router.route(tok, ids, w)
    x2, _ = exact_data(T, H, E, 22)
    tok.copy_(to_bf16(x2))
    graph.replay()
    torch.cuda.synchronize()
    assert np.array_equal(ids.cpu().numpy(), sublayer.choose(x2 @ g.T, k))
