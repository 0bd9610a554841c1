"""zipmoe_add_rmsnorm where the norm has no finite value: eps = 0 and a sum of squares that is zero or lies below the smallest
normal number of fp32.  What the header says of such rows, and that their neighbours are not touched."""
import numpy as np
import pytest

from paper_2601_21198_b200 import build

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [512, 500, 20000])
def test_rows_without_a_norm(cols):
    import torch
    build.build()
    from paper_2601_21198_b200 import binding as zb
    x = torch.randn(4, cols, device="cuda")
    x[0] = 0
    x[1] = 1e-24
    x[1, 7] = 0
    x[2] = 1e-12                               # far above: an ordinary row
    x = x.to(torch.bfloat16)
    w = torch.ones(cols, dtype=torch.bfloat16, device="cuda")
    out = zb.RmsNorm(w, 0.0).add_norm(x).float().cpu().numpy()
    assert np.isnan(out[0]).all()
    assert np.isnan(out[1, 7]) and np.isposinf(np.delete(out[1], 7)).all()
    assert np.abs(out[2] - 1).max() <= 2.0 ** -8 + 2e-5 and np.isfinite(out[3]).all()
    for group in (0, 128):
        q, s = zb.RmsNorm(w, 0.0).add_norm_8bit(x, group=group)
        s = s.cpu().numpy()
        assert np.isnan(s[0]).all() and not np.isfinite(s[1, 0]) and np.isfinite(s[2:]).all()
    eps = zb.RmsNorm(w, 1e-12)
    out = eps.add_norm(x).float().cpu().numpy()
    q, s = eps.add_norm_8bit(x, group=128)
    assert not out[0].any() and np.abs(out[1]).max() < 1e-17 and np.isfinite(out).all()
    assert not q.float()[0].any() and not s[0].any()
