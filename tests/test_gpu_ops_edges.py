"""Calls of the operators that users may make and the other tests do not: refused
ones, several at once, tensors that are passed twice, many heads on one key head."""
import pytest

from tests.test_gpu_window import CASES, check_backward, check_forward, expect, make, sentinels

pytestmark = pytest.mark.gpu

import paper_2609_25869_amd as bsa  # noqa: E402  (fails loudly if the libraries are missing)


def test_refusals_of_the_binding():
    import torch
    z = lambda *s, dtype=torch.bfloat16: torch.zeros(s, dtype=dtype, device="cuda")
    q, k, lse = z(2, 6, 4, 64), z(2, 9, 2, 64), z(2, 4, 6, dtype=torch.float32)
    i32 = torch.zeros(2, dtype=torch.int32, device="cuda")
    fwd = lambda **kw: bsa.window_forward(**{**dict(q=q, k=k, v=k, left=3), **kw})
    bwd = lambda **kw: bsa.window_backward(**{**dict(q=q, k=k, v=k, o=z(2, 6, 4, 64), lse=lse, do=q, left=3), **kw})
    bad = [(fwd, dict(scale=1e-50), ValueError), (fwd, dict(scale=0.0), ValueError), (fwd, dict(scale=float("nan")), ValueError),
           (fwd, dict(k=k.cpu()), TypeError), (fwd, dict(v=k.half()), TypeError), (fwd, dict(v=k[:, :8]), ValueError),
           (fwd, dict(q=q[0]), ValueError), (fwd, dict(q=q[..., ::2]), ValueError), (fwd, dict(k=k[:1]), ValueError),
           (fwd, dict(q=z(2, 6, 3, 64)), bsa.BsaError), (fwd, dict(q=q.float(), k=k.float(), v=k.float()), bsa.BsaError),
           (fwd, dict(q=q[..., :32], k=k[..., :32], v=k[..., :32]), bsa.BsaError), (fwd, dict(left=-2), bsa.BsaError),
           (fwd, dict(q_len=i32.long()), TypeError), (fwd, dict(kv_len=i32[:1]), ValueError), (fwd, dict(o=q), bsa.BsaError),
           (fwd, dict(o=q[:1].expand(2, -1, -1, -1)), bsa.BsaError), (fwd, dict(lse=lse[:, :, :5]), TypeError),
           (fwd, dict(q=z(2, 6, 4, 72)[..., 1:65]), bsa.BsaError), (bwd, dict(dq=q), bsa.BsaError),
           (bwd, dict(dk=z(2, 9, 2, 64)[:, :8]), ValueError), (bwd, dict(lse=lse.double()), TypeError),
           (bwd, dict(workspace=z(16)), bsa.BsaError), (bwd, dict(do=q[..., :1].expand(2, 6, 4, 64)), ValueError)]
    for call, kw, error in bad:
        with pytest.raises(error):
            call(**kw)
    freq = bsa.rope_frequencies((16, 16))
    rope = lambda **kw: bsa.rope(**{**dict(q=q, freq=freq, pairs=(16, 16), grid=(2, 3, 1)), **kw})
    p = torch.zeros((2, 2, 6), dtype=torch.int32, device="cuda")
    for kw, error in [(dict(freq=freq.float()), TypeError), (dict(freq=freq[:31]), TypeError), (dict(pairs=(16, 17)), TypeError),
                      (dict(grid=None), ValueError), (dict(positions=p), ValueError), (dict(rows=i32), ValueError),
                      (dict(grid=None, positions=p[:1]), ValueError), (dict(grid=None, positions=p.long()), TypeError),
                      (dict(grid=None, positions=p[:, :, :5]), ValueError), (dict(v=k), ValueError),
                      (dict(grid=(0, 1, 1)), bsa.BsaError), (dict(k=k), ValueError), (dict(out_q=q[:, :, :3]), ValueError),
                      (dict(k=q, out_k=q, out_q=q), bsa.BsaError)]:
        with pytest.raises(error):
            rope(**kw)


def test_calls_at_once():
    """Two streams at a time over the same inputs, with workspaces and results of
    their own."""
    import torch
    made = [make(c, "bf16", seed=11) for c in ("one_token_long_split", "sinks_wide")]
    call = lambda x, lens, win, **kw: (lambda f: f + bsa.window_backward(
        x["q"], x["k"], x["v"], f[0], f[1], x["do"], *win, **lens, **kw))(
            bsa.window_forward(x["q"], x["k"], x["v"], *win, **lens, **kw))
    alone = [call(*m[:3]) for m in made]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    for _ in range(3):
        out = [call(*made[i % 2][:3], stream=s) for i, s in enumerate(streams)]
        torch.cuda.synchronize()
        for i, o in enumerate(out):
            assert all(torch.equal(a, b) for a, b in zip(o, alone[i % 2])), i


@pytest.mark.parametrize("d", [64, 128])
def test_one_tensor_as_q_k_and_v(d):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    x = torch.randn((2, 200, 3, d), generator=g, device="cuda").bfloat16()
    do = torch.randn(x.shape, generator=g, device="cuda").bfloat16()
    o, lse = bsa.window_forward(x, x, x, 40, 0, 2)
    got = (o, lse) + bsa.window_backward(x, x, x, o, lse, do, 40, 0, 2)
    y = [x.clone() for _ in range(3)]
    o, lse = bsa.window_forward(*y, 40, 0, 2)
    want = (o, lse) + bsa.window_backward(*y, o, lse, do, 40, 0, 2)
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_everything_in_place_on_a_side_stream():
    import torch
    pairs = (10, 11, 11)
    freq = bsa.rope_frequencies(pairs)
    qkv = torch.randn((3, 33, 6, 64), device="cuda").half()
    before, q, k, v = qkv.clone(), qkv[:, :, :3], qkv[:, :, 3:5], qkv[:, :, 5:]
    v = v.expand(-1, -1, 2, -1).contiguous()
    kept = v.clone()
    lengths = torch.tensor([33, 0, 7], dtype=torch.int32, device="cuda")
    kw = dict(freq=freq, pairs=pairs, grid=(2, 4, 4), origin=(5, -2, 1))
    want = bsa.rope(before[:, :, :3], before[:, :, 3:5], **kw)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    bsa.rope(q, k, v, out_q=q, out_k=k, out_v=v, lengths=lengths, stream=side, **kw)
    side.synchronize()
    assert torch.equal(v, kept) and torch.equal(qkv[:, :, 5:], before[:, :, 5:])
    for b, n in enumerate((33, 0, 7)):
        for got, turned, old in ((q, want[0], before[:, :, :3]), (k, want[1], before[:, :, 3:5])):
            assert torch.equal(got[b, :n], turned[b, :n]) and torch.equal(got[b, n:], old[b, n:])


@pytest.mark.parametrize("name,case", [
    ("many_heads_on_one", (1, 256, 1, 1, 2600, 64, -1, 0, 0, None, None)),
    ("many_heads_few_keys", (2, 160, 1, 3, 70, 128, 5, 1, 2, [3, 2], [70, 1])),
])
def test_many_heads_on_one_key_head(name, case, monkeypatch):
    import torch
    monkeypatch.setitem(CASES, name, case)
    x, lens, win, clipped = make(name, "bf16", seed=12)
    r = expect(x, win, clipped)
    o, lse, dq, dk, dv = sentinels(x)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse, **lens)
    bsa.window_backward(x["q"], x["k"], x["v"], o, lse, x["do"], *win, dq=dq, dk=dk, dv=dv, **lens)
    torch.cuda.synchronize()
    check_forward(o, lse, r, "bf16", name)
    check_backward(dq, dk, dv, r, "bf16", name)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name,case", [
    ("uneven_ragged", (3, 4, 2, 300, 300, 128, -1, 0, 0, [300, 1, 130], [300, 40, 131])),
    ("uneven_right", (2, 3, 3, 260, 260, 64, 0, -1, 0, None, [260, 100])),
    ("uneven_long_axis", (3, 4, 2, 40, 3001, 128, -1, 0, 5, [40, 3, 0], [3001, 2000, 10])),
    ("uneven_sinks", (2, 6, 3, 700, 700, 128, 400, 0, 130, [700, 513], [700, 513])),
])
def test_walks_of_uneven_length(name, case, dtype, monkeypatch):
    """Tiles that are dealt out, longest first, over sequences of several lengths."""
    import torch
    monkeypatch.setitem(CASES, name, case)
    x, lens, win, clipped = make(name, dtype, seed=13)
    r = expect(x, win, clipped)
    o, lse, dq, dk, dv = sentinels(x)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse, **lens)
    bsa.window_backward(x["q"], x["k"], x["v"], o, lse, x["do"], *win, dq=dq, dk=dk, dv=dv, **lens)
    torch.cuda.synchronize()
    check_forward(o, lse, r, dtype, name)
    check_backward(dq, dk, dv, r, dtype, name)
