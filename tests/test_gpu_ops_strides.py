"""Strides of axes of length 1 on the device."""
import pytest

from tests.test_gpu_window import sentinels

pytestmark = pytest.mark.gpu

import paper_2609_25869_amd as bsa  # noqa: E402  (fails loudly if the libraries are missing)


@pytest.mark.parametrize("token", [0, 1 << 23, 1 << 31, 1 << 40])
@pytest.mark.parametrize("nq,nkv", [(1, 1), (1, 70), (70, 1)])
@pytest.mark.parametrize("d", [64, 128])
def test_token_stride_of_one_token(d, nq, nkv, token):
    """Tensors of one token give the same bits whatever their token stride is: 2^31 elements are
    2^32 bytes, which is 0 in 32 bits."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    x = {n: torch.randn((2, s, h, d), generator=g, device="cuda").bfloat16()
         for n, s, h in (("q", nq, 4), ("k", nkv, 2), ("v", nkv, 2), ("do", nq, 4))}
    far = lambda t: t.as_strided(t.shape, (t.stride(0), token, d, 1)) if t.shape[1] == 1 else t
    got = []
    for y in (x, {n: far(t) for n, t in x.items()}):
        o, lse, dq, dk, dv = sentinels(x)
        bsa.window_forward(y["q"], y["k"], y["v"], -1, -1, o=o, lse=lse)
        bsa.window_backward(y["q"], y["k"], y["v"], o, lse, y["do"], -1, -1, dq=dq, dk=dk, dv=dv)
        got.append((o, lse, dq, dk, dv))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))
