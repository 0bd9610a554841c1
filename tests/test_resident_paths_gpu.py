"""Paths of zipmoe_expert_ffn that small layers do not reach: experts taken in two groups (from 450 MB of active weights, or 1 GB
where an expert has more than 72 tokens), the combination of five to eight choices of many tokens, and, for up to 8 tokens,
the whole-rows kernel's handling of choices that are no expert, repeated experts, NaN and infinities.  Against the formula
in fp64 (computed on the device for the large layers), with every output held to a bound from its own terms: one rounding of h
to bf16 (half a step, 2^(e - 8) in [2^e, 2^(e+1)), which reaches the output through |w| |W2|; the kernels keep more of it), one
of the output, and the fp32 sums contribute 2e-6 of the sum of the magnitudes they add."""
import numpy as np
import pytest

from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def half_step(v):
    import torch
    return torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -126))) - 8)


def layer(E, H, I, seed):
    """3 * E bf16 tensors in arrays of one kind, standard deviation 1 / sqrt(columns)."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    kinds = []
    for rows, cols in ((I, H), (I, H), (H, I)):
        w = torch.empty(E, rows, cols, dtype=torch.bfloat16, device="cuda")
        for e in range(E):
            w[e] = torch.randn(rows, cols, generator=g, device="cuda") / cols ** 0.5
        kinds.append(w)
    return [kinds[j][e] for e in range(E) for j in range(3)]


def tokens_of(T, H, seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16)


def check(y, ws, x, ids, wts):
    """ids [T, k], wts [T, k] or None: numpy arrays."""
    import torch
    E = len(ws) // 3
    out, slack = torch.zeros(x.shape, dtype=torch.float64, device="cuda"), torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    for e in range(E):
        t = np.nonzero((ids == e).any(axis=1))[0]
        if not t.size:
            continue
        share = ((ids[t] == e) * (1.0 if wts is None else wts[t].astype(np.float64))).sum(axis=1)
        share = torch.from_numpy(share).cuda()[:, None]
        t = torch.from_numpy(t).cuda()
        xt = x[t].double()
        w1, w3, w2 = (ws[3 * e + j].double() for j in range(3))
        g, u = xt @ w1.t(), xt @ w3.t()
        s = g / (1 + torch.exp(-g))
        h = s * u
        off = 2e-6 * ((xt.abs() @ w1.abs().t()) * 1.1 * u.abs() + (xt.abs() @ w3.abs().t()) * s.abs())
        out[t] += share * (h @ w2.t())
        slack[t] += share.abs() * ((half_step(h) + h.abs() * 4e-6 + off) @ w2.abs().t())
    bound = half_step(out) + out.abs() * 1e-5 + slack + 1e-30
    off = ((y.double() - out).abs() / bound).max().item()
    assert off <= 1, off


def routing(T, k, active, seed):
    """Ids [T, k], k distinct ones of `active` per token, and weights."""
    rng = np.random.default_rng(seed)
    ids = np.stack([rng.permutation(np.asarray(active))[:k] for _ in range(T)]).astype(np.int32)
    return ids, rng.random((T, k)).astype(np.float32) + 0.1


def run(ex, x, ids, wts):
    import torch
    return ex.ffn(x, torch.from_numpy(ids).cuda(), None if wts is None else torch.from_numpy(wts).cuda())


# (bytes of an expert are 6 * hidden * inter; `active` of `E` experts have tokens)
@pytest.mark.parametrize("E,H,I,T,k,active", [
    (1, 8192, 9344, 9, 1, [0]),                  # 459 MB, one expert: the second group is empty
    (2, 6144, 6400, 12, 2, [0, 1]),              # 472 MB, one expert in each
    (5, 4096, 6424, 16, 2, [0, 2, 4]),           # 474 MB, two and one, rows and columns behind the last whole 64
    (4, 4096, 4928, 16, 3, [0, 1, 2, 3]),        # 484 MB, two experts in each
    (16, 2056, 2312, 40, 6, range(16)),          # 456 MB, top-6: tokens packed, up to 8 lanes per output
    (2, 8192, 10432, 90, 1, [0, 1]),             # 1.03 GB with more than 72 tokens of one expert
    (3, 8192, 7184, 200, 2, [0, 1, 2]),          # 1.06 GB, shares by weight, the widest operand
])
def test_two_groups_of_experts(zb, E, H, I, T, k, active):
    import torch
    active = list(active)
    ws = layer(E, H, I, E + T)
    ex = zb.ResidentExperts(ws, H, I)
    x = tokens_of(T, H, T)
    ids, wts = routing(T, k, active, T)
    if T == 90:                                  # 73 tokens and 17
        ids[:, 0] = np.where(np.arange(T) < 73, 0, 1)
    assert sorted(set(ids.ravel())) == active
    most = max((ids == e).any(axis=1).sum() for e in active)
    assert len(active) * 6 * H * I >= (1000000000 if most > 72 else 450000000)
    first = run(ex, x, ids, wts)
    check(first, ws, x, ids, wts)
    # one group (fewer experts), few tokens and two groups again, all on one workspace
    if len(active) > 1:
        one = np.full_like(ids, active[-1])
        check(run(ex, x, one, wts), ws, x, one, wts)
    check(run(ex, x[:3], ids[:3], wts[:3]), ws, x[:3], ids[:3], wts[:3])
    assert torch.equal(run(ex, x, ids, wts), first)
    check(run(ex, x, ids, None), ws, x, ids, None)
    assert int(ex.status.item()) == 0


def test_two_groups_of_scattered_experts_with_choices_that_do_not_count(zb):
    import torch
    E, H, I, T, k = 5, 4096, 4928, 24, 4
    ws = layer(E, H, I, 3)
    apart = [w.clone() for w in ws[::-1]][::-1]
    ex = zb.ResidentExperts(apart, H, I)
    x = tokens_of(T, H, 5)
    ids, wts = routing(T, k, range(E), 7)
    ids[3], ids[4, 1:], ids[6] = -1, -1, [1, 0, 1, -7]
    ids[T - 1] = [4, 3, 2, 0]
    y = run(ex, x, ids, wts)
    check(y, ws, x, ids, wts)
    assert not y[3].any() and int(ex.status.item()) == 0
    assert torch.equal(y, run(zb.ResidentExperts(ws, H, I), x, ids, wts))


@pytest.mark.parametrize("E,H,I,T,k", [(16, 1024, 768, 64, 6), (9, 2056, 328, 33, 5), (32, 512, 256, 200, 8), (8, 264, 200, 256, 7)])
def test_five_to_eight_choices_of_many_tokens(zb, E, H, I, T, k):
    """Where T x hidden is beyond 56832 every thread adds up to eight choices of a token."""
    assert T * H > 56832
    ws = layer(E, H, I, k)
    ex = zb.ResidentExperts(ws, H, I)
    x = tokens_of(T, H, 1)
    ids, wts = routing(T, k, range(E), 2)
    check(run(ex, x, ids, wts), ws, x, ids, wts)
    check(run(ex, x, ids, None), ws, x, ids, None)
    ids[1], ids[2, 1:], ids[5, :2], ids[7, -1] = -1, -1, ids[5, 2], -9
    y = run(ex, x, ids, wts)
    check(y, ws, x, ids, wts)
    assert not y[1].any() and int(ex.status.item()) == 0


SMALL = [(5, 256, 320, 4), (6, 264, 200, 3), (4, 1096, 904, 4), (7, 520, 72, 3)]      # experts, hidden, inter, choices


@pytest.mark.parametrize("E,H,I,k", SMALL)
@pytest.mark.parametrize("T", [1, 2, 5, 8, 9, 24])
def test_empty_rows_and_repeated_experts(zb, E, H, I, k, T):
    ws = layer(E, H, I, 70 + T)
    ex = zb.ResidentExperts(ws, H, I)
    x = tokens_of(T, H, T)
    ids, wts = routing(T, k, range(E), T)
    ids[T // 2] = -1                       # a token without any expert
    ids[0] = [2] * k                       # one expert with all of a token's choices
    if T > 2:
        ids[1, 1:] = -1
        ids[T - 1, :3] = [1, 0, 1]
    y = run(ex, x, ids, wts)
    check(y, ws, x, ids, wts)
    assert T == 1 or not y[T // 2].any()
    none = np.full_like(ids, -1)
    none[T // 2, 0] = -(2 ** 31)
    assert not run(ex, x, none, wts).any() and int(ex.status.item()) == 0
    every = np.zeros_like(ids)             # all choices of all tokens on one expert
    check(run(ex, x, every, wts), ws, x, every, wts)
    check(run(ex, x, ids, None), ws, x, ids, None)
    assert int(ex.status.item()) == 0
    ids[0, 0], ids[T - 1, -1] = E, 2 ** 31 - 1
    check(run(ex, x, ids, wts), ws, x, ids, wts)
    assert int(ex.status.item()) == 1


@pytest.mark.parametrize("E,H,I,k", SMALL)
@pytest.mark.parametrize("T", [4, 8, 17])
def test_infinities_and_nan_stay_where_they_belong(zb, E, H, I, k, T):
    """A token with NaN, and experts with infinite weights, touch only the tokens that meet them - also what lay in shared
    memory and in the workspace before a sound call."""
    import torch
    ws = layer(E, H, I, 90)
    x = tokens_of(T, H, 8)
    rng = np.random.default_rng(T)
    ids = np.stack([rng.permutation(np.arange(E - 2)) for _ in range(T)])[:, :2].astype(np.int32)   # the last two experts are poisoned
    ids[1], ids[2] = [E - 1, 0], [E - 2, 1]
    wts = rng.random(ids.shape).astype(np.float32) + 0.1
    poisoned, bad = [w.clone() for w in ws], x.clone()
    bad[0, H - 3] = float("nan")
    poisoned[3 * (E - 1) + 2][9, I - 1] = float("inf")
    poisoned[3 * (E - 2) + 0][I - 2, H - 1] = float("-inf")
    ex = zb.ResidentExperts(poisoned, H, I)
    got = run(ex, bad, ids, wts)
    assert got[0].isnan().all()
    assert not torch.isfinite(got[1, 9]) and torch.isfinite(got[1, torch.arange(H, device="cuda") != 9]).all()
    assert not torch.isfinite(got[2]).all()
    clean = list(range(3, T))
    check(got[clean], ws, x[clean], ids[clean], wts[clean])
    # a sound call after it, with fewer tokens
    check(run(ex, x[clean], ids[clean], wts[clean]), ws, x[clean], ids[clean], wts[clean])
    # every row, column and token poisoned, then a sound call of other experts
    for w in poisoned[3 * (E - 1):]:
        w.fill_(float("nan"))
    run(ex, torch.full_like(x, float("nan")), np.full_like(ids, E - 1), wts)
    check(run(ex, x[clean], ids[clean], wts[clean]), ws, x[clean], ids[clean], wts[clean])
    assert int(ex.status.item()) == 0
