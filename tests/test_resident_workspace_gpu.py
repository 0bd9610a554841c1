"""The scratch that ResidentExperts keeps for zipmoe_expert_ffn: calls captured into graphs, on several streams and by
several layers never share a workspace that is not theirs, nor meet one that was not prepared.  Every output is compared bit
for bit with the same call outside of any graph (the kernels give the same bits whatever the timing)."""
import numpy as np
import pytest

from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu
E, H, I, K = 6, 512, 384, 3


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def dev(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a.view(np.int16) if a.dtype == np.uint16 else a)).cuda()


@pytest.fixture(scope="module")
def weights():
    return [dev(inputs.gaussian((I, H) if j % 3 < 2 else (H, I), 0.05, 300 + j)) for j in range(3 * E)]


def call(T):
    """Inputs of one call and an output that holds what no call writes."""
    import torch
    ids, wts = inputs.routing(T, n_experts=E, k=K, seed=T)
    return dev(inputs.tokens(T, H, seed=T)), dev(ids), dev(wts), torch.full((T, H), 0x5555, dtype=torch.int16, device="cuda")


def capture(ex, args, stream=None):
    import torch
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        ex.ffn(*args)
    return graph


@pytest.mark.parametrize("sizes", [(1, 2), (40, 3), (2, 200), (200, 40)])     # both kernels, tokens gathered and packed
def test_graphs_without_a_call_before_them_replayed_in_any_order(zb, weights, sizes):
    import torch
    ex = zb.ResidentExperts(weights, H, I)
    calls = [call(T) for T in sizes]
    graphs = [capture(ex, c) for c in calls]
    graphs[1].replay()
    graphs[0].replay()
    graphs[1].replay()
    torch.cuda.synchronize()
    assert int(ex.status.item()) == 0
    other = zb.ResidentExperts(weights, H, I)
    for c in calls:
        assert torch.equal(c[3], other.ffn(*c[:3]))


def test_a_call_on_the_capturing_stream_before_the_first_replay(zb, weights):
    import torch
    ex = zb.ResidentExperts(weights, H, I)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph_args, args = call(20), call(20)
    graph = capture(ex, graph_args, side)
    ex.ffn(*args, stream=side)
    side.synchronize()
    assert int(ex.status.item()) == 0
    graph.replay()
    torch.cuda.synchronize()
    want = zb.ResidentExperts(weights, H, I).ffn(*args[:3])
    assert torch.equal(args[3], want) and torch.equal(graph_args[3], want) and int(ex.status.item()) == 0
    del graph            # its memory may go to somebody else: the stream's own workspace must not be in it
    torch.cuda.empty_cache()
    junk = [torch.full((1 << 20,), 0x77777777, dtype=torch.int32, device="cuda") for _ in range(64)]
    args[3].fill_(0x5555)
    side.wait_stream(torch.cuda.current_stream())
    ex.ffn(*args, stream=side)
    side.synchronize()
    assert torch.equal(args[3], want) and int(ex.status.item()) == 0
    del junk


def test_more_tokens_within_one_capture(zb, weights):
    """A capture whose later call wants a larger workspace than its first, the stream having one of its own already."""
    import torch
    ex = zb.ResidentExperts(weights, H, I)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    calls = [call(T) for T in (5, 129, 40)]
    with torch.cuda.stream(side):
        ex.ffn(*calls[0][:3])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        for c in calls:
            ex.ffn(*c)
    with torch.cuda.stream(side):       # between the capture and its replay, with more tokens than before
        between = ex.ffn(*calls[1][:3])
    graph.replay()
    torch.cuda.synchronize()
    assert int(ex.status.item()) == 0
    other = zb.ResidentExperts(weights, H, I)
    assert torch.equal(between, other.ffn(*calls[1][:3]))
    for c in calls:
        assert torch.equal(c[3], other.ffn(*c[:3]))
    for _ in range(3):
        for c in calls:
            c[3].fill_(0x5555)
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(c[3], other.ffn(*c[:3])) for c in calls) and int(ex.status.item()) == 0


def test_graphs_replayed_on_two_streams_do_not_meet(zb, weights):
    """Two graphs captured one after the other on one stream, then replayed with no order between them, beside calls
    outside of any graph: each has a workspace of its own."""
    import torch
    ex = zb.ResidentExperts(weights, H, I)
    calls = [call(T) for T in (3, 60, 130)]
    graphs = [capture(ex, c) for c in calls[:2]]
    sides = [torch.cuda.Stream(), torch.cuda.Stream()]
    want = [zb.ResidentExperts(weights, H, I).ffn(*c[:3]) for c in calls]
    torch.cuda.synchronize()
    for _ in range(20):
        for c in calls:
            c[3].fill_(0x5555)
        for s, g in zip(sides, graphs):
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                for _ in range(5):
                    g.replay()
        ex.ffn(*calls[2])
        torch.cuda.synchronize()
        assert all(torch.equal(c[3], w) for c, w in zip(calls, want))
    assert int(ex.status.item()) == 0


def held_for(fn):
    """Device memory that is in use after fn() beyond what was in use before, and what it returned."""
    import gc
    import torch
    gc.collect()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    kept = fn()
    gc.collect()
    torch.cuda.synchronize()
    return torch.cuda.memory_allocated() - before, kept


def test_scratch_is_one_workspace_per_stream_whatever_the_batches_and_layers(zb, weights):
    import torch
    T_max = 256
    tok, ids = torch.zeros(T_max, H, dtype=torch.int16, device="cuda"), torch.zeros(T_max, K, dtype=torch.int32, device="cuda")
    out = torch.empty(T_max, H, dtype=torch.int16, device="cuda")
    first = zb.ResidentExperts(weights, H, I)
    largest = zb.zipmoe_expert_ffn_workspace_bytes(T_max, K, first.struct)

    def rising(ex):
        for T in list(range(1, 17)) + list(range(17, 129, 13)) + list(range(129, T_max + 1)):
            ex.ffn(tok[:T], ids[:T], None, out[:T])

    def other_layers():
        layers = [zb.ResidentExperts(weights, H, I) for _ in range(5)]
        for ex in layers:
            rising(ex)
        return layers

    of_one, _ = held_for(lambda: rising(first))
    assert largest <= of_one <= largest + (2 << 20)
    of_more, layers = held_for(other_layers)
    assert of_more <= 1 << 20                                    # their tables and status words
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())

    def on_another_stream():
        with torch.cuda.stream(side):
            rising(first)
            rising(layers[0])
        side.synchronize()

    of_stream, _ = held_for(on_another_stream)
    assert largest <= of_stream <= largest + (2 << 20)
    assert int(first.status.item()) == 0 and all(int(ex.status.item()) == 0 for ex in layers)


def test_scratch_is_given_back_with_the_last_layer(zb, weights):
    import torch

    def life():
        ex = zb.ResidentExperts(weights, H, I)
        T = 200
        ex.ffn(torch.zeros(T, H, dtype=torch.int16, device="cuda"), torch.zeros(T, K, dtype=torch.int32, device="cuda"), None)
        torch.cuda.synchronize()
        del ex

    of_life, _ = held_for(life)
    assert of_life <= 0


def test_layers_of_different_sizes_share_a_workspace(zb):
    """Calls of a large and a small layer in turn, few tokens and many: each leaves the workspace ready for the other."""
    import torch
    layers = []
    for E2, H2, I2 in ((6, 512, 384), (3, 264, 1000)):
        ws = [dev(inputs.gaussian((I2, H2) if j % 3 < 2 else (H2, I2), 0.05, 700 + j)) for j in range(3 * E2)]
        calls = []
        for T in (5, 130, 30, 2):
            ids, wts = inputs.routing(T, n_experts=E2, k=2, seed=T)
            calls.append((dev(inputs.tokens(T, H2, seed=T)), dev(ids), dev(wts)))
        layers.append((zb.ResidentExperts(ws, H2, I2), calls))
    want = [[ex.ffn(*c) for c in calls] for ex, calls in layers]
    for _ in range(3):
        for i in range(4):
            for (ex, calls), w in zip(layers, want):
                assert torch.equal(ex.ffn(*calls[i]), w[i])
    assert all(int(ex.status.item()) == 0 for ex, _ in layers)


def test_a_decode_step_of_several_layers_in_one_graph(zb, weights):
    """Norm, router and experts of three layers, captured without a call before it, replayed on new inputs: the launches that
    are set up while their predecessors drain keep their order inside a graph too."""
    import torch
    T = 7
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    bf16 = dict(dtype=torch.bfloat16, device="cuda")
    layers = [(zb.RmsNorm((1 + 0.1 * torch.randn(H, generator=g, device="cuda")).to(torch.bfloat16)),
               zb.Router((0.05 * torch.randn(E, H, generator=g, device="cuda")).to(torch.bfloat16), K),
               zb.ResidentExperts(weights, H, I)) for _ in range(3)]
    x, residual = torch.zeros(T, H, **bf16), torch.zeros(T, H, **bf16)

    def step(x, residual):
        for norm, router, experts in layers:
            h = norm.add_norm(x, residual, residual)
            ids, wts = router.route(h)
            x = experts.ffn(h, ids, wts)
        return x

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y = step(x, residual)
    for _ in range(10):
        new_x, new_residual = (torch.randn(T, H, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        x.copy_(new_x)
        residual.copy_(new_residual)
        graph.replay()
        want = step(new_x, new_residual)
        assert torch.equal(y, want) and torch.equal(residual, new_residual)
    assert all(int(router.status.item()) == 0 and int(experts.status.item()) == 0 for _, router, experts in layers)
