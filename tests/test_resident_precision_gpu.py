"""zipmoe_expert_ffn keeps 16 significant bits of h between the two products: an output is off by its own rounding to bf16 and
hardly more.  Bounds from the terms of every output, in fp64: h in two bf16 parts is off by 2^-16 of itself at most, the fp32
sums and SiLU add 4e-6 of the magnitudes they add (2e-6 through g and u), and the output's own rounding is half a step of the
value that those errors can move it to."""
import numpy as np
import pytest

from paper_2601_21198_b200 import build

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def half_step(v):
    import torch
    return torch.exp2(torch.floor(torch.log2(v.clamp(min=2.0 ** -126))) - 8)


def layer(E, H, I, seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [(torch.randn(I if j < 2 else H, H if j < 2 else I, generator=g, device="cuda") / (H if j < 2 else I) ** 0.5).to(torch.bfloat16)
            for _ in range(E) for j in range(3)]


def expected(ws, x, ids, wts):
    """(out, how far a value may be off before its own rounding), fp64."""
    import torch
    out, off = (torch.zeros(x.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    for e in range(len(ws) // 3):
        t, j = torch.nonzero(ids == e, as_tuple=True)
        if not t.numel():
            continue
        xt = x[t].double()
        w1, w3, w2 = (w.double() for w in ws[3 * e:3 * e + 3])
        g, u = xt @ w1.t(), xt @ w3.t()
        s = g / (1 + torch.exp(-g))
        h = s * u
        from_sums = 2e-6 * ((xt.abs() @ w1.abs().t()) * 1.1 * u.abs() + (xt.abs() @ w3.abs().t()) * s.abs())
        share = wts[t, j].double()[:, None]
        out.index_add_(0, t, share * (h @ w2.t()))
        off.index_add_(0, t, share * ((h.abs() * (2.0 ** -16 + 4e-6) + from_sums) @ w2.abs().t()))
    return out, off + out.abs() * 1e-6 + 1e-30


@pytest.mark.parametrize("E,H,I,k", [(6, 512, 384, 2), (9, 264, 200, 3), (4, 1096, 904, 1), (5, 2056, 72, 4)])
@pytest.mark.parametrize("T", [1, 4, 5, 8, 9, 16, 37, 100, 130, 256])
def test_outputs_are_off_by_their_own_rounding(zb, T, E, H, I, k):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    ws = layer(E, H, I, T + H)
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    ids = torch.rand(T, E, generator=g, device="cuda").argsort(dim=1)[:, :k].to(torch.int32)
    wts = torch.rand(T, k, generator=g, device="cuda") + 0.1
    ex = zb.ResidentExperts(ws, H, I)
    got = ex.ffn(x, ids, wts).double()
    out, off = expected(ws, x, ids, wts)
    worst = ((got - out).abs() / (half_step(out.abs() + off) + off)).max().item()
    assert worst <= 1, worst
    # in the mean: no further off than the formula rounded once (an unrounded h would be)
    once = (out.to(torch.bfloat16).double() - out).norm()
    assert (got - out).norm() <= 1.05 * once + off.norm()
    assert int(ex.status.item()) == 0


def test_experts_with_many_tokens_beside_others_with_few(zb):
    """Shares by weight, the widest operand and the narrowest in one call; top-1 of a few experts, 240 tokens on one."""
    import torch
    E, H, I, T = 7, 1024, 1416, 256
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    ws = layer(E, H, I, 5)
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    for most in (256, 240, 130, 73, 50, 37):
        ids = torch.full((T, 1), 3, dtype=torch.int32, device="cuda")
        rest = T - most
        ids[most:, 0] = torch.arange(rest, device="cuda", dtype=torch.int32) % (E - 1)
        wts = torch.ones(T, 1, device="cuda")
        ex = zb.ResidentExperts(ws, H, I)
        got = ex.ffn(x, ids, wts).double()
        out, off = expected(ws, x, ids, wts)
        assert ((got - out).abs() <= half_step(out.abs() + off) + off).all(), most
        assert int(ex.status.item()) == 0


@pytest.mark.parametrize("T", [1, 6, 40, 200])
def test_infinite_weights_and_activations_give_infinities(zb, T):
    """W2 with an infinite weight, and g so large that h leaves fp32: the formula's infinities, with their signs."""
    import torch
    E, H, I = 1, 128, 192
    g = torch.Generator(device="cuda")
    g.manual_seed(T)
    ws = layer(E, H, I, 17)
    x = torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)
    ids, wts = torch.zeros(T, 1, dtype=torch.int32, device="cuda"), torch.ones(T, 1, device="cuda")
    sound, _ = expected(ws, x, ids, wts)
    h = (lambda a, b: a / (1 + torch.exp(-a)) * b)(x.double() @ ws[0].double().t(), x.double() @ ws[1].double().t())
    ws[2][7, 100] = float("inf")
    got = zb.ResidentExperts(ws, H, I).ffn(x, ids, wts).double()
    assert torch.equal(got[:, 7], torch.sign(h[:, 100]) * float("inf"))
    rest = torch.arange(H, device="cuda") != 7
    assert torch.isfinite(got[:, rest]).all() and (got - sound)[:, rest].norm() <= 0.01 * sound.norm()
    # h beyond fp32 in one place: every output is that place's weight times infinity
    ws[2][7, 100] = 1.0
    ws[0][50], ws[1][50] = 0, 0
    ws[0][50, 0], ws[1][50, 0] = 1e30, 1e30
    x[:, 0] = 1.0
    got = zb.ResidentExperts(ws, H, I).ffn(x, ids, wts).double()
    assert torch.equal(got, torch.sign(ws[2][:, 50].double()).expand_as(got) * float("inf"))
