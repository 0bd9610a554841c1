"""zipmoe_expert_ffn (experts recovered to bf16) on the GPU against the formula in fp64.  Every output is held to a bound
from its own terms: h is rounded to bf16 (by half a step of bf16 at most, 2^(e - 8) in [2^e, 2^(e+1)), which reaches the
output through |w| |W2|), the output once more, and the fp32 sums contribute 2e-6 of the sum of the magnitudes they add."""
import numpy as np
import pytest

from oracle.ffn import bf16_to_f64, silu
from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def half_step(v):
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - 8)


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a.view(np.int16) if a.dtype == np.uint16 else a)).cuda()


def layer(E, H, I, seed, std=0.05):
    return [inputs.gaussian((I, H) if j < 2 else (H, I), std * (1 + 0.3 * ((e + j) % 3)), seed + 3 * e + j)
            for e in range(E) for j in range(3)]


def expected(ws, tok, ids, wts):
    """(out, bound) in float64: the formula, and how far a correct implementation may be from it."""
    x = bf16_to_f64(tok)
    out, slack = np.zeros(x.shape), np.zeros(x.shape)
    for e in sorted(set(int(i) for i in ids.ravel() if 0 <= i < len(ws) // 3)):
        w1, w3, w2 = (bf16_to_f64(ws[3 * e + j]) for j in range(3))
        t = np.nonzero((ids == e).any(axis=1))[0]
        share = ((ids[t] == e) * (1.0 if wts is None else wts[t].astype(np.float64))).sum(axis=1)[:, None]
        g, u = x[t] @ w1.T, x[t] @ w3.T
        h = silu(g) * u
        off = 2e-6 * ((np.abs(x[t]) @ np.abs(w1).T) * 1.1 * np.abs(u) + (np.abs(x[t]) @ np.abs(w3).T) * np.abs(silu(g)))
        out[t] += share * (h @ w2.T)
        slack[t] += np.abs(share) * ((half_step(h) + np.abs(h) * 4e-6 + off) @ np.abs(w2).T)
    return out, half_step(out) + np.abs(out) * 1e-5 + slack + 1e-30


def check(y, ws, tok, ids, wts):
    import torch
    torch.cuda.synchronize()
    got = bf16_to_f64(y.view(torch.int16).cpu().numpy().view(np.uint16))
    want, bound = expected(ws, tok, ids, wts)
    assert got.shape == want.shape
    assert (np.abs(got - want) <= bound).all(), float((np.abs(got - want) / bound).max())


@pytest.mark.parametrize("T", [1, 2, 7, 16, 17, 33, 64, 65, 128, 200, 256])
@pytest.mark.parametrize("E,H,I,k", [(4, 512, 768, 2), (9, 264, 200, 3)])
def test_batches(zb, T, E, H, I, k):
    ws = layer(E, H, I, 900 + E)
    ex = zb.ResidentExperts([dev(w) for w in ws], H, I)
    tok = inputs.tokens(T, H, seed=T)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=T)
    for w in (wts, None):
        y = ex.ffn(dev(tok), dev(ids), None if w is None else dev(w))
        check(y, ws, tok, ids, w)
    assert int(ex.status.item()) == 0


@pytest.mark.parametrize("E,H,I,k,T", [(1, 8, 8, 1, 1), (1, 8, 8, 1, 3), (2, 64, 128, 1, 5), (3, 128, 64, 2, 4), (2, 1000, 24, 2, 9),
                                       (2, 24, 1000, 2, 9), (64, 256, 136, 8, 31), (256, 64, 40, 8, 256), (2, 2048, 1408, 1, 3),
                                       (2, 1416, 2056, 2, 2), (1, 4096, 4096, 1, 1), (3, 16384, 256, 1, 2), (3, 256, 16384, 2, 2)])
def test_shapes(zb, E, H, I, k, T):
    ws = layer(E, H, I, 40 + E, std=1.0 / np.sqrt(max(H, I)))
    ex = zb.ResidentExperts([dev(w) for w in ws], H, I)
    tok = inputs.tokens(T, H, seed=E)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=I)
    check(ex.ffn(dev(tok), dev(ids), dev(wts)), ws, tok, ids, wts)
    assert int(ex.status.item()) == 0


@pytest.mark.parametrize("E,H,I,k,T", [(1, 8192, 1024, 1, 3), (1, 16384, 512, 1, 2), (1, 8200, 1032, 1, 8), (2, 4096, 4104, 2, 8),
                                       (2, 5120, 1536, 1, 5)])
def test_few_tokens_through_several_sets_of_rows(zb, E, H, I, k, T):
    """A block's rows of W1 and W3 beyond 16, of W2 beyond 32, come in several sets."""
    ws = layer(E, H, I, 60 + E, std=1.0 / np.sqrt(max(H, I)))
    ex = zb.ResidentExperts([dev(w) for w in ws], H, I)
    tok = inputs.tokens(T, H, seed=E)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=I)
    check(ex.ffn(dev(tok), dev(ids), dev(wts)), ws, tok, ids, wts)
    assert int(ex.status.item()) == 0


def test_empty_rows_and_repeated_experts(zb):
    """Ids of -1 (a router with experts switched off), tokens without any expert, an expert listed twice."""
    E, H, I, T, k = 5, 256, 320, 40, 4
    ws = layer(E, H, I, 70)
    ex = zb.ResidentExperts([dev(w) for w in ws], H, I)
    tok = inputs.tokens(T, H, seed=2)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=2)
    ids[3] = -1
    ids[4, 2:] = -1
    ids[5] = [2, 2, 2, 2]
    ids[6] = [1, 0, 1, -5]
    y = ex.ffn(dev(tok), dev(ids), dev(wts))
    check(y, ws, tok, ids, wts)
    assert not y[3].any() and int(ex.status.item()) == 0
    ids[:] = -1
    assert not ex.ffn(dev(tok), dev(ids), dev(wts)).any()
    assert int(ex.status.item()) == 0
    every = np.zeros((T, k), np.int32)       # all choices of all tokens on one expert
    check(ex.ffn(dev(tok), dev(every), dev(wts)), ws, tok, every, wts)


def test_ids_out_of_range_are_reported_and_add_nothing(zb):
    E, H, I, T, k = 3, 128, 128, 6, 2
    ws = layer(E, H, I, 7)
    ex = zb.ResidentExperts([dev(w) for w in ws], H, I)
    tok = inputs.tokens(T, H, seed=1)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=1)
    ids[2, 1], ids[4, 0] = E, 2 ** 31 - 1
    check(ex.ffn(dev(tok), dev(ids), dev(wts)), ws, tok, ids, wts)
    assert int(ex.status.item()) == 1


def test_infinities_and_nan_stay_where_they_belong(zb):
    """A token with NaN, and an expert with an infinite weight, touch only the tokens that meet them."""
    E, H, I, T, k = 4, 128, 192, 24, 2
    ws = layer(E, H, I, 31)
    tok = inputs.tokens(T, H, seed=8)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=8)
    tok[5, 17] = 0x7FC0
    ws[3 * 3 + 2][9, 100] = 0x7F80        # w2 of expert 3, output column 9
    ws[3 * 2 + 0][50, 60] = 0xFF80        # w1 of expert 2
    y = zb.ResidentExperts([dev(w) for w in ws], H, I).ffn(dev(tok), dev(ids), dev(wts))
    got = bf16_to_f64(y.cpu().numpy().view(np.uint16))
    clean = [t for t in range(T) if t != 5 and 2 not in ids[t]]
    with_3 = [t for t in clean if 3 in ids[t]]
    assert with_3 and len(with_3) < len(clean)
    assert np.isnan(got[5]).all()
    assert not np.isfinite(got[with_3][:, 9]).any()
    cols = np.arange(H) != 9
    good = layer(E, H, I, 31)
    tok[5, 17] = 0
    want, bound = expected(good, tok, ids, wts)
    assert (np.abs(got - want) <= bound)[np.ix_(clean, cols)].all()
    alone = [t for t in clean if 3 not in ids[t]]
    assert (np.abs(got - want) <= bound)[alone].all()


def test_decoded_experts_are_run_where_they_lie(zb):
    """zipmoe_decode's output buffer goes straight in, and gives what the fused call on the compressed experts gives."""
    import torch
    E, H, I, T, k = 3, 512, 768, 11, 2
    ws = layer(E, H, I, 210, std=0.03)
    blobs = [zb.zipmoe_encode(w, layout=zb.LAYOUT_BLOCKED, chunk_elems=65536) for w in ws]
    plan = zb.DecodePlan(blobs)
    dv = plan.to_device("cuda")
    buf = dv.new_output()
    dv.decode(buf)
    tok = inputs.tokens(T, H, seed=3)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=3)
    y = zb.ResidentExperts.from_decode(plan, buf, H, I).ffn(dev(tok), dev(ids), dev(wts))
    check(y, ws, tok, ids, wts)
    fused = zb.DeviceExperts(blobs, H, I).ffn(dev(tok), dev(ids), dev(wts))
    a, b = y.view(torch.bfloat16).float(), fused.view(torch.bfloat16).float()
    assert ((a - b).abs() <= torch.maximum(torch.full_like(b, 1e-2), b.abs() * 2.0 ** -7)).all()


def test_the_same_bits_again_and_on_another_stream(zb):
    """No atomics on values: the result does not depend on which block finishes first; calls follow each other on one
    workspace, and two streams have workspaces of their own."""
    import torch
    E, H, I, T, k = 8, 1024, 1408, 48, 4
    ws = layer(E, H, I, 5)
    ex = zb.ResidentExperts([dev(w) for w in ws], H, I)
    tok, (ids, wts) = inputs.tokens(T, H, seed=4), inputs.routing(T, n_experts=E, k=k, seed=4)
    tok_d, ids_d, wts_d = dev(tok), dev(ids), dev(wts)
    first = ex.ffn(tok_d, ids_d, wts_d)
    for T2 in (1, 48, 5, 48):
        again = ex.ffn(tok_d[:T2].contiguous(), ids_d[:T2].contiguous(), wts_d[:T2].contiguous())
        if T2 == T:
            assert torch.equal(again, first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    outs = []
    for i in range(10):
        outs.append(ex.ffn(tok_d, ids_d, wts_d, stream=side if i % 2 else None))
    torch.cuda.synchronize()
    assert all(torch.equal(o, first) for o in outs)
    check(first, ws, tok, ids, wts)


def test_captured_into_a_graph(zb):
    import torch
    E, H, I, T, k = 6, 512, 384, 12, 3
    ws = layer(E, H, I, 15)
    ex = zb.ResidentExperts([dev(w) for w in ws], H, I)
    tok, (ids, wts) = inputs.tokens(T, H, seed=4), inputs.routing(T, n_experts=E, k=k, seed=4)
    tok_d, ids_d, wts_d = dev(tok), dev(ids), dev(wts)
    out = torch.empty(T, H, dtype=torch.int16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        ex.ffn(tok_d, ids_d, wts_d, out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ex.ffn(tok_d, ids_d, wts_d, out)
    tok2, (ids2, wts2) = inputs.tokens(T, H, seed=14), inputs.routing(T, n_experts=E, k=k, seed=14)
    for d, n in ((tok_d, tok2), (ids_d, ids2), (wts_d, wts2)):
        d.copy_(dev(n))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    check(out, ws, tok2, ids2, wts2)


def test_no_tokens(zb):
    import torch
    ws = layer(1, 64, 64, 1)
    ex = zb.ResidentExperts([dev(w) for w in ws], 64, 64)
    y = ex.ffn(torch.empty(0, 64, dtype=torch.int16, device="cuda"), torch.empty(0, 1, dtype=torch.int32, device="cuda"), None)
    assert y.shape == (0, 64)


def test_binding_refuses_what_the_kernel_would_misread(zb):
    import torch
    ws = [dev(w) for w in layer(2, 64, 64, 1)]
    ex = zb.ResidentExperts(ws, 64, 64)
    t, i = torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, 1, dtype=torch.int32, device="cuda")
    for bad in ((t.half(), i, None), (t, i.long(), None), (t[:, :32], i, None), (t, i, torch.ones(3, 2, device="cuda")),
                (t.cpu(), i, None), (t, i, torch.ones(3, 1, device="cuda").half())):
        with pytest.raises(ValueError):
            ex.ffn(*bad)
    with pytest.raises(zb.ZipMoEError):
        ex.ffn(torch.zeros(257, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(257, 1, dtype=torch.int32, device="cuda"), None)
    with pytest.raises(ValueError):
        zb.ResidentExperts(ws[:4], 64, 64)
    with pytest.raises(ValueError):
        zb.ResidentExperts(ws, 64, 72)


@pytest.mark.parametrize("E,H,I,k", [(5, 512, 384, 2), (4, 264, 200, 3), (1, 128, 64, 1)])
@pytest.mark.parametrize("T", [3, 40])
def test_evenly_spaced_and_scattered_experts_give_the_same_bits(zb, E, H, I, k, T):
    """Tensors at equal distances are found through one map per kind, others through the table."""
    import torch
    ws = layer(E, H, I, 77)
    tok, (ids, wts) = inputs.tokens(T, H, seed=4), inputs.routing(T, n_experts=E, k=k, seed=4)
    stacked = [torch.stack([dev(ws[3 * e + j]) for e in range(E)]) for j in range(3)]
    even = zb.ResidentExperts([stacked[j][e] for e in range(E) for j in range(3)], H, I)
    assert even.struct.even == 1
    a = even.ffn(dev(tok), dev(ids), dev(wts))
    check(a, ws, tok, ids, wts)
    if E == 1:
        return
    room = torch.zeros(3 * E * (H * I + 8) + 8, dtype=torch.int16, device="cuda")
    at = {int(s): 8 * i + i * H * I for i, s in enumerate(np.random.default_rng(1).permutation(3 * E)[::-1])}
    scattered = []
    for s in range(3 * E):
        view = room[at[s]:at[s] + H * I].view(ws[s].shape)
        view.copy_(dev(ws[s]))
        scattered.append(view)
    apart = zb.ResidentExperts(scattered, H, I)
    assert apart.struct.even == 0
    b = apart.ffn(dev(tok), dev(ids), dev(wts))
    assert torch.equal(a, b) and int(apart.status.item()) == 0 and int(even.status.item()) == 0
