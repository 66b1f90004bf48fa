"""Values of V that are not finite, on the device: what reaches the queries that see
them, where their weight leaves 32 bits, and what that costs."""
import numpy as np
import pytest

from tests.test_gpu_window import f64

pytestmark = pytest.mark.gpu

import paper_2609_25869_amd as bsa  # noqa: E402  (fails loudly if the libraries are missing)

INF, NAN = float("inf"), float("nan")


@pytest.mark.parametrize("bad", [INF, -INF, NAN])
@pytest.mark.parametrize("d,heads", [(64, 1), (128, 1), (64, 8), (128, 8)])
def test_slices_without_weight_keep_what_is_not_finite(d, heads, bad):
    """One token over keys in slices.  The scores of the first 2000 keys lie 40 sqrt(d) below
    the others', a weight that 32 bits hold as 0 beside them: a slice of such keys alone still
    hands on a value that is not finite."""
    import torch
    q = torch.full((1, 1, heads, d), 4.0, device="cuda").bfloat16()
    k = torch.zeros((1, 4000, 1, d), device="cuda").bfloat16()
    k[:, :2000] = -10.0
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    v = torch.randn((1, 4000, 1, d), generator=g, device="cuda").bfloat16()
    want = bsa.window_forward(q, k, v, -1)[0]
    assert bsa.window_workspace(q, k, v, -1) > 0
    v[0, 100, 0, 7] = bad
    o = bsa.window_forward(q, k, v, -1)[0]
    torch.cuda.synchronize()
    hit = f64(o)[..., 7]
    assert np.all(np.isnan(hit) if np.isnan(bad) else hit == bad)
    rest = [c for c in range(d) if c != 7]
    assert torch.equal(o[..., rest], want[..., rest])
