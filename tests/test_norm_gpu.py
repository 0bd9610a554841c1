"""zipmoe_add_rmsnorm on the GPU against the fp64 oracle.  Tolerances: one rounding to bf16 is half of the step between
its neighbours, 2^(e - 8) for a value of [2^e, 2^(e+1)) (8 significant bits); the arithmetic before it is fp32 with at most a few thousand terms in the sum of squares, whose error is a relative error of
the whole row far below 2e-5 (pairwise-summed positive terms).  An e4m3 value is within 2^-4 of its real number, or half
of the smallest step 2^-9 times the scale."""
import numpy as np
import pytest

from oracle import sublayer
from oracle.ffn import bf16_to_f64
from paper_2601_21198_b200 import build, inputs

pytestmark = pytest.mark.gpu
FP32 = 2e-5


def half_step(v):
    """Half of the distance between neighbouring bf16 values around v: the most that a rounding may move it."""
    return np.exp2(np.floor(np.log2(np.maximum(np.abs(v), 2.0 ** -126))) - 8)


@pytest.fixture(scope="module")
def zb():
    build.build()
    from paper_2601_21198_b200 import binding
    return binding


def rows_apart(bits, pitch, dev_dtype):
    """Device view [rows, cols] of a numpy array, rows `pitch` elements apart, the gaps filled with a marker."""
    import torch
    rows, cols = bits.shape
    wide = np.full((rows, pitch), 0x55, bits.dtype)
    wide[:, :cols] = bits
    return torch.from_numpy(wide).cuda().view(dev_dtype)[:, :cols]


def bf16(t):
    import torch
    return bf16_to_f64(t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16))


def run(zb, rows, cols, pitch, residual, group, seed, want_out=True):
    """One call; returns everything as float64 together with the oracle's values."""
    import torch
    rng = np.random.default_rng(seed)
    xb = inputs.f32_to_bf16_bits(rng.standard_normal((rows, cols)).astype(np.float32))
    wb = inputs.f32_to_bf16_bits((1 + 0.3 * rng.standard_normal(cols)).astype(np.float32))
    x = rows_apart(xb.view(np.int16), pitch, torch.bfloat16)
    r = r64 = None
    if residual == "f32":
        rb = (3 * rng.standard_normal((rows, cols))).astype(np.float32)
        r, r64 = rows_apart(rb, pitch, torch.float32), rb.astype(np.float64)
    elif residual == "bf16":
        rb = inputs.f32_to_bf16_bits((3 * rng.standard_normal((rows, cols))).astype(np.float32))
        r, r64 = rows_apart(rb.view(np.int16), pitch, torch.bfloat16), bf16_to_f64(rb)
    norm = zb.RmsNorm(torch.from_numpy(wb.view(np.int16)).cuda(), 1e-5)
    r_out = None if r is None else torch.empty(rows, cols, dtype=r.dtype, device="cuda")
    got = {}
    if group is None:
        got["out"] = bf16(norm.add_norm(x, r, r_out))
    else:
        out = torch.empty(rows, cols, dtype=torch.bfloat16, device="cuda") if want_out else None
        q, s = norm.add_norm_8bit(x, r, r_out, group=group, out=out)
        got["q"], got["s"] = sublayer.e4m3_to_f64(q.view(torch.uint8).cpu().numpy()), s.cpu().numpy().astype(np.float64)
        if want_out:
            got["out"] = bf16(out)
    if r_out is not None:
        got["residual"] = bf16(r_out) if residual == "bf16" else r_out.cpu().numpy().astype(np.float64)
    h, y = sublayer.add_rmsnorm(bf16_to_f64(xb), r64, bf16_to_f64(wb), 1e-5)
    return got, h, y


def check(got, h, y, residual, group):
    tiny = 1e-38
    if "out" in got:
        assert (np.abs(got["out"] - y) <= half_step(y) + np.abs(y) * FP32 + tiny).all()
    if residual == "bf16":
        assert (np.abs(got["residual"] - h) <= half_step(h) + np.abs(h) * FP32 + tiny).all()
    elif residual == "f32":
        assert (np.abs(got["residual"] - h) <= np.abs(h) * 2.0 ** -24 + tiny).all()
    if group is not None:
        want = sublayer.group_scales(y, group)
        assert got["s"].shape == want.shape
        assert (np.abs(got["s"] - want) <= want * FP32 + tiny).all()
        cols = y.shape[1]
        g = cols if group <= 0 or group >= cols else group
        s = np.repeat(got["s"], g, axis=1)[:, :cols]
        assert (np.abs(got["q"] * s - y) <= np.maximum(np.abs(y) * 2.0 ** -4, s * 2.0 ** -10) * 1.001 + np.abs(y) * FP32).all()


@pytest.mark.parametrize("residual", ["none", "bf16", "f32"])
@pytest.mark.parametrize("rows,cols,pitch", [(1, 8, 8), (1, 2048, 2048), (3, 1408, 1416), (2, 1, 1), (5, 7, 9), (4, 333, 333),
                                             (3, 257, 300), (2, 4096, 4096), (2, 4097, 4097), (1, 14336, 14336),
                                             (2, 16400, 16400), (1, 32768, 32768), (2, 32761, 32765), (300, 96, 104)])
def test_bf16_rows(zb, rows, cols, pitch, residual):
    got, h, y = run(zb, rows, cols, pitch, residual, None, rows * 7 + cols)
    check(got, h, y, residual, None)


@pytest.mark.parametrize("group", [0, 32, 64, 128, 256])
@pytest.mark.parametrize("rows,cols,pitch,residual", [(1, 2048, 2048, "bf16"), (3, 1408, 1416, "f32"), (2, 40, 48, "none"),
                                                      (7, 333, 340, "bf16"), (2, 4100, 4100, "f32"), (2, 14336, 14336, "bf16"),
                                                      (1, 32767, 32767, "none"), (129, 128, 128, "bf16")])
def test_8bit_rows(zb, rows, cols, pitch, residual, group):
    got, h, y = run(zb, rows, cols, pitch, residual, group, rows + cols + group, want_out=group != 64)
    check(got, h, y, residual, group)


def test_alignment_of_every_pointer(zb):
    """Rows that start at odd elements: sliced columns of a wider tensor."""
    import torch
    rng = np.random.default_rng(5)
    rows, cols = 6, 1000
    for shift in (1, 2, 3, 5, 8):
        wide = torch.from_numpy(rng.standard_normal((rows, 1024)).astype(np.float32)).cuda().to(torch.bfloat16)
        x, w = wide[:, shift:shift + cols], wide[0, :cols].clone()
        out = torch.zeros(rows, 1024, dtype=torch.bfloat16, device="cuda")
        zb.RmsNorm(w, 1e-6).add_norm(x, out=out[:, shift:shift + cols])
        _, y = sublayer.add_rmsnorm(bf16(x), None, bf16(w), 1e-6)
        got = bf16(out)
        assert (np.abs(got[:, shift:shift + cols] - y) <= half_step(y) + np.abs(y) * FP32 + 1e-38).all(), shift
        assert not got[:, :shift].any() and not got[:, shift + cols:].any(), "written outside the rows"


def test_in_place(zb):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn(33, 2048, generator=g, device="cuda").to(torch.bfloat16)
    r = torch.randn(33, 2048, generator=g, device="cuda").to(torch.bfloat16)
    norm = zb.RmsNorm(torch.ones(2048, dtype=torch.bfloat16, device="cuda"))
    r2 = torch.empty_like(r)
    want = norm.add_norm(x, r, r2)
    x_in, r_in = x.clone(), r.clone()
    norm.add_norm(x_in, r_in, r_in, out=x_in)
    assert torch.equal(x_in, want) and torch.equal(r_in, r2)


def test_rows_of_zeros_infinities_and_nan(zb):
    import torch
    cols = 512
    x = torch.randn(6, cols, device="cuda")
    x[0] = 0
    x[1, 3] = float("inf")
    x[2, 4] = float("nan")
    x[3] = 3e38            # the sum of squares leaves fp32: zeros, as documented
    x[4] = 1e-30           # far below eps
    x = x.to(torch.bfloat16)
    norm = zb.RmsNorm(torch.ones(cols, dtype=torch.bfloat16, device="cuda"), 1e-6)
    out = norm.add_norm(x).float().cpu().numpy()
    assert not out[0].any() and not out[3].any()
    assert np.isnan(out[1, 3]) and not np.delete(out[1], 3).any()
    assert np.isnan(out[2]).all()
    want = bf16(x)[4] / 1e-3
    assert (np.abs(out[4] - want) <= half_step(want) + np.abs(want) * FP32).all()
    assert np.isfinite(out[5]).all()
    for group in (0, 128):
        q, s = norm.add_norm_8bit(x, group=group)
        q, s = q.float().cpu().numpy(), s.cpu().numpy()
        assert not q[0].any() and not s[0].any()
        assert np.isnan(s[1, 0]) and np.isnan(s[2]).all() and not s[3].any() and not q[3].any()
        assert np.isfinite(q[5]).all() and (np.abs(q[5]).max() == 448)


def test_no_rows_and_another_stream(zb):
    import torch
    w = torch.ones(256, dtype=torch.bfloat16, device="cuda")
    norm = zb.RmsNorm(w)
    assert norm.add_norm(torch.empty(0, 256, dtype=torch.bfloat16, device="cuda")).shape == (0, 256)
    side = torch.cuda.Stream()
    x = torch.randn(2000, 256, device="cuda").to(torch.bfloat16)
    want = norm.add_norm(x)
    side.wait_stream(torch.cuda.current_stream())
    got = norm.add_norm(x, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_binding_refuses_what_the_kernel_would_misread(zb):
    import torch
    norm = zb.RmsNorm(torch.ones(64, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        norm.add_norm(torch.zeros(2, 64, dtype=torch.float16, device="cuda"))
    with pytest.raises(ValueError):
        norm.add_norm(torch.zeros(2, 63, dtype=torch.bfloat16, device="cuda"))
    with pytest.raises(ValueError):
        norm.add_norm(torch.zeros(64, 2, dtype=torch.bfloat16, device="cuda").t())
    with pytest.raises(ValueError):
        norm.add_norm(torch.zeros(2, 64, dtype=torch.bfloat16))
    with pytest.raises(zb.ZipMoEError):
        norm.add_norm_8bit(torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda"), group=48)
