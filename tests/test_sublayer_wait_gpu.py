"""A wait that runs out in the router or the expert FFN ends in a status word, not in a hang: the library's test switch arms
the barriers of their copies for more bytes than the copies deliver and shortens the waits, so that the barriers never
complete although every copy lands.  The calls after it are exact again: nothing is left behind in the workspace."""
import numpy as np
import pytest

from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a.view(np.int16) if a.dtype == np.uint16 else a)).cuda()


@pytest.mark.parametrize("T", [1, 5, 40, 200])     # both kernels, tokens gathered and packed
def test_expert_ffn(zb, T):
    import torch
    E, H, I, k = 4, 512, 384, 2
    ex = zb.ResidentExperts([dev(inputs.gaussian((I, H) if j % 3 < 2 else (H, I), 0.05, 60 + j)) for j in range(3 * E)], H, I)
    ids, wts = inputs.routing(T, n_experts=E, k=k, seed=T)
    args = dev(inputs.tokens(T, H, seed=T)), dev(ids), dev(wts)
    want = ex.ffn(*args)
    torch.cuda.synchronize()
    assert int(ex.status.item()) == 0
    zb.zipmoe_test_wait_fault(16, 64)
    try:
        ex.ffn(*args)
        torch.cuda.synchronize()
    finally:
        zb.zipmoe_test_wait_fault(0, 0)
    assert int(ex.status.item()) == 3
    ex.status.zero_()
    for _ in range(2):
        assert torch.equal(ex.ffn(*args), want)
    assert int(ex.status.item()) == 0


@pytest.mark.parametrize("T", [1, 300])
def test_router(zb, T):
    import torch
    E, H, k = 64, 1024, 6
    router = zb.Router(dev(inputs.gaussian((E, H), 0.02, 5)), k)
    x = dev(inputs.tokens(T, H, seed=T))
    want = router.route(x)
    torch.cuda.synchronize()
    assert int(router.status.item()) == 0
    zb.zipmoe_test_wait_fault(16, 64)
    try:
        router.route(x)
        torch.cuda.synchronize()
    finally:
        zb.zipmoe_test_wait_fault(0, 0)
    assert int(router.status.item()) == 3
    router.status.zero_()
    got = router.route(x)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1]) and int(router.status.item()) == 0


def test_a_workspace_that_was_not_prepared_is_reported(zb):
    import torch
    E, H, I, T, k = 2, 128, 128, 3, 1
    ex = zb.ResidentExperts([dev(inputs.gaussian((H, I), 0.05, j)) for j in range(3 * E)], H, I)
    tok, ids = dev(inputs.tokens(T, H, seed=1)), torch.zeros(T, k, dtype=torch.int32, device="cuda")
    for T2 in (3, 40):
        tok2, ids2 = tok[:1].repeat(T2, 1), ids[:1].repeat(T2, 1)
        n2 = zb.zipmoe_expert_ffn_workspace_bytes(T2, k, ex.struct)
        ws = torch.zeros(n2, dtype=torch.uint8, device="cuda")
        out = torch.full((T2, H), 0x5555, dtype=torch.int16, device="cuda")
        stream = torch.cuda.current_stream().cuda_stream
        zb.zipmoe_expert_ffn(tok2, T2, ids2, None, k, ex.struct, out, ws, n2, ex.status, stream)
        torch.cuda.synchronize()
        assert int(ex.status.item()) == 1 and bool((out == 0x5555).all())
        ex.status.zero_()
        zb.zipmoe_expert_ffn_workspace_init(ws, n2, stream)
        zb.zipmoe_expert_ffn(tok2, T2, ids2, None, k, ex.struct, out, ws, n2, ex.status, stream)
        assert torch.equal(out, ex.ffn(tok2, ids2, None)) and int(ex.status.item()) == 0
