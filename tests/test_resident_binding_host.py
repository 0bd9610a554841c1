"""What the binding's classes for the expert sublayer do on the host: no GPU is needed (addresses are never followed)."""
import pytest

from paper_2601_21198_b200 import build


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def test_capture_id_wants_somewhere_to_put_it(zb):
    assert zb._lib.zipmoe_stream_capture_id(None, None) == zb.ERR_INVALID_ARG


class FakeTensor:
    """What the binding asks a dense tensor for, without a device."""

    def __init__(self, shape, dtype, index):
        import torch
        self.shape, self.dtype, self.index, self.device = torch.Size(shape), dtype, index, torch.device("cpu")

    def get_device(self):
        return self.index

    def stride(self):
        return tuple(int(self.shape[i + 1:].numel()) for i in range(len(self.shape)))

    def is_contiguous(self):
        return True

    def numel(self):
        return self.shape.numel()

    def data_ptr(self):
        return 1 << 20


class FakeDevices:
    """Two devices, the first of them current; records which one was current when the library was called."""

    def __init__(self, zb, monkeypatch):
        import torch
        self.current, self.seen = 0, []
        kinds = zb._Kinds()
        kinds.current_device = lambda: self.current
        kinds.current_stream = lambda index: 0          # (the default stream has this handle on every device)
        kinds.capturing = lambda: False
        monkeypatch.setattr(zb, "_kinds", kinds)
        devices = self

        class Guard:
            def __init__(self, index):
                self.index = index

            def __enter__(self):
                self.before, devices.current = devices.current, self.index

            def __exit__(self, *_):
                devices.current = self.before

        monkeypatch.setattr(torch.cuda, "device", Guard)

        def called(name, result):
            def fn(*_):
                self.seen.append((name, self.current))
                return result
            return fn

        for name in ("zipmoe_add_rmsnorm", "zipmoe_route", "zipmoe_expert_ffn", "zipmoe_expert_ffn_workspace_init"):
            monkeypatch.setattr(zb._lib, name, called(name, 0))

        def plan(tensors, n_experts, hidden, inter):
            import numpy as np
            self.seen.append(("plan", self.current))
            return np.zeros(3 * n_experts * zb.RESIDENT_ENTRY_BYTES, np.uint8), zb.ResidentExpertsStruct(n_experts, hidden, inter)

        monkeypatch.setattr(zb, "zipmoe_resident_experts_plan", plan)


class FakeStream:
    def __init__(self, index):
        self.device_index, self.cuda_stream = index, 5


def calls_on_device_1(zb):
    import torch
    def t(*shape, dtype=torch.bfloat16):
        return FakeTensor(shape, dtype, 1)

    norm = zb.RmsNorm(t(64))
    router = zb.Router(t(8, 64), 2)
    experts = zb.ResidentExperts([t(64, 64) for _ in range(6)], 64, 64)
    ids, wts = t(3, 2, dtype=torch.int32), t(3, 2, dtype=torch.float32)
    return (lambda stream=None: norm.add_norm(t(3, 64), out=t(3, 64), stream=stream),
            lambda stream=None: router.route(t(3, 64), ids, wts, stream=stream),
            lambda stream=None: experts.ffn(t(3, 64), ids, wts, t(3, 64), stream=stream))


def test_calls_are_made_with_their_tensors_device_current(zb, monkeypatch):
    devices = FakeDevices(zb, monkeypatch)
    for call in calls_on_device_1(zb):
        call()
    names = [name for name, _ in devices.seen]
    assert names == ["plan", "zipmoe_add_rmsnorm", "zipmoe_route", "zipmoe_expert_ffn_workspace_init", "zipmoe_expert_ffn"]
    assert [current for _, current in devices.seen] == [1] * 5 and devices.current == 0


def test_streams_of_another_device_are_refused(zb, monkeypatch):
    devices = FakeDevices(zb, monkeypatch)
    calls = calls_on_device_1(zb)
    del devices.seen[:]
    for call in calls:
        with pytest.raises(ValueError):
            call(stream=FakeStream(0))
    assert not devices.seen


@pytest.mark.parametrize("grid", [0, 1, 1 << 30])
def test_a_plan_for_a_device_of_another_size_is_refused(zb, grid):
    """The boxes that a plan's tensor maps bring in follow the number of SMs: a call that takes other boxes would wait for
    bytes that never come.  (No device has one SM or none of them, so nothing is launched here, wherever this runs.)"""
    A = 1 << 20
    for T in (4, 40):
        ex = zb.ResidentExpertsStruct(4, 64, 128, 0, A)
        ex.grid = grid
        n = zb.zipmoe_expert_ffn_workspace_bytes(T, 2, ex)
        with pytest.raises(zb.ZipMoEError) as err:
            zb.zipmoe_expert_ffn(A, T, A, A, 2, ex, A, A, n)
        assert err.value.status == zb.ERR_INVALID_ARG


def test_experts_of_another_orientation_are_refused(zb, monkeypatch):
    """w1 and w3 are [inter, hidden] and w2 is [hidden, inter]: a matrix the other way round has as many elements and would
    be read as something else.  Flat tensors (slices of a decode launch's output) have no orientation."""
    import torch
    devices = FakeDevices(zb, monkeypatch)
    hidden, inter = 64, 128

    def tensors(change=None):
        shapes = [(inter, hidden), (inter, hidden), (hidden, inter)] * 2
        if change is not None:
            shapes[change] = shapes[change][::-1]
        return [FakeTensor(s, torch.bfloat16, 0) for s in shapes]

    zb.ResidentExperts(tensors(), hidden, inter)
    zb.ResidentExperts([FakeTensor((hidden * inter,), torch.int16, 0) for _ in range(6)], hidden, inter)
    del devices.seen[:]
    for i in range(6):
        with pytest.raises(ValueError):
            zb.ResidentExperts(tensors(i), hidden, inter)
    with pytest.raises(ValueError):
        zb.ResidentExperts([FakeTensor((4, hidden * inter // 4), torch.bfloat16, 0)] + tensors()[1:], hidden, inter)
    assert not devices.seen
