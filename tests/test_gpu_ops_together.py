"""The operators in the runs they are made for: a stream that is prompted and then
extended token by token, a training step through rotation and attention, and the
rotation in front of the block-sparse request path."""
import numpy as np
import pytest

from oracle import rope as orope
from oracle import window as owin
from tests import test_gpu_window as tw

pytestmark = pytest.mark.gpu

import paper_2609_25869_amd as bsa  # noqa: E402  (fails loudly if the libraries are missing)


def normal(g, *shape):
    import torch
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def test_prompt_then_tokens_over_a_cache():
    """Two streams of different lengths: the cache filled by the prompt's rotated keys, then
    three rounds of new tokens appended and attended, against one whole-sequence oracle."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    B, H, Hkv, d, cap, left, sinks = 2, 8, 2, 128, 220, 60, 3
    pairs, n_prompt, rounds = (32, 16, 16), [150, 97], [1, 1, 4]
    freq = bsa.rope_frequencies(pairs, shared=True)
    total = sum(rounds)
    whole = max(n_prompt) + total
    q, k, v = normal(g, B, whole, H, d), normal(g, B, whole, Hkv, d), normal(g, B, whole, Hkv, d)
    pos = torch.randint(0, 5000, (3, B, whole), generator=g, device="cuda", dtype=torch.int32)
    ck = torch.full((B, cap, Hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    cv = ck.clone()
    i32 = lambda l: torch.tensor(l, dtype=torch.int32, device="cuda")

    # the prompt, padded to the longer one
    N = max(n_prompt)
    rq, *_ = bsa.rope(q[:, :N], k[:, :N], v[:, :N], freq=freq, pairs=pairs, positions=pos[:, :, :N].contiguous(),
                      interleaved=False, lengths=i32(n_prompt), rows=i32([0, 0]), out_k=ck, out_v=cv)
    outs = [[], []]
    o, lse = bsa.window_forward(rq, ck, cv, left, 0, sinks, q_len=i32(n_prompt), kv_len=i32(n_prompt))
    for b in range(B):
        outs[b].append((o[b, :n_prompt[b]], lse[b, :, :n_prompt[b]]))
    done = list(n_prompt)
    for n in rounds:
        take = lambda t: torch.stack([t[b, done[b]:done[b] + n] for b in range(B)])
        p = torch.stack([pos[:, b, done[b]:done[b] + n] for b in range(B)], 1).contiguous()
        rq, *_ = bsa.rope(take(q), take(k), take(v), freq=freq, pairs=pairs, positions=p, interleaved=False,
                          rows=i32(done), out_k=ck, out_v=cv)
        done = [x + n for x in done]
        o, lse = bsa.window_forward(rq, ck, cv, left, 0, sinks, kv_len=i32(done))
        for b in range(B):
            outs[b].append((o[b], lse[b]))
    torch.cuda.synchronize()
    for b in range(B):
        L = done[b]
        turn = lambda t: orope.rotate(tw.f64(t[b, :L]), pos[:, b].cpu().numpy(), freq.cpu().numpy(), pairs, False)
        # the kernels round the rotated tensors to bf16: so does the oracle's input
        bf = lambda a: torch.from_numpy(a).to(torch.bfloat16).double().numpy()[None]
        r = owin.window_attention(bf(turn(q)), bf(turn(k)), tw.f64(v[b, :L])[None], left, 0, sinks)
        o = torch.cat([x[0] for x in outs[b]])[None]
        lse = torch.cat([x[1] for x in outs[b]], 1)[None]
        e = r["err"]
        # a rotated value next to a rounding border may fall to the other side: 2^-7 of it, in
        # few of them; 1% of the weights' sum covers one such value in every score
        tol = 1.01 * tw.U["bf16"] * (e["o_u"] + np.abs(r["o"])) + 1e-2 * e["o_u"]
        tw.close("o", o, r["o"], tol)
        tw.close("lse", lse, r["lse"], 1e-2)


def test_gradients_through_rotation_and_attention():
    """d(sum(O * g)) of O = attention(rope(q), rope(k), v): backward, then the inverse rotation,
    against directional differences of the oracle in 64 bits."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    B, N, H, Hkv, d, left, right, sinks = 1, 48, 4, 2, 64, 12, 3, 2
    pairs, grid = (10, 11, 11), (3, 4, 4)
    freq = bsa.rope_frequencies(pairs)
    t = torch.float16
    q, k, v = (torch.randn((B, N, h, d), generator=g, device="cuda").to(t) for h in (H, Hkv, Hkv))
    do = torch.randn(q.shape, generator=g, device="cuda").to(t)
    rq, rk = bsa.rope(q, k, freq=freq, pairs=pairs, grid=grid)
    o, lse = bsa.window_forward(rq, rk, v, left, right, sinks)
    drq, drk, dv = bsa.window_backward(rq, rk, v, o, lse, do, left, right, sinks)
    dq, dk = bsa.rope(drq, drk, freq=freq, pairs=pairs, grid=grid, inverse=True)
    torch.cuda.synchronize()
    pos, _ = orope.grid_positions(N, grid)
    turn = lambda a: orope.rotate(a[0], pos, freq.cpu().numpy(), pairs, True)[None]
    x = dict(q=tw.f64(q), k=tw.f64(k), v=tw.f64(v))
    got = dict(q=tw.f64(dq), k=tw.f64(dk), v=tw.f64(dv))

    def loss(y):
        return float((owin.window_attention(turn(y["q"]), turn(y["k"]), y["v"], left, right, sinks)["o"] * tw.f64(do)).sum())

    rng = np.random.default_rng(5)
    for name in "qkv":
        for _ in range(3):
            way = rng.standard_normal(x[name].shape)
            h = 1e-4
            diff = (loss({**x, name: x[name] + h * way}) - loss({**x, name: x[name] - h * way})) / (2 * h)
            # six roundings of 2^-11 on the way (rotated tensors, P, dS, O in D, the gradient, its
            # rotation), each of terms up to twice the gradient's size: a vector of errors below
            # 2^-7 of the gradient's norm, of which a normal direction sees four sigma at most
            tol = 4 * 2.0 ** -7 * np.linalg.norm(got[name])
            assert abs(float((got[name] * way).sum()) - diff) < tol, name


def test_rotation_before_a_block_sparse_request():
    """rope -> sparsify -> plan -> forward on the device equals the same request on tensors that
    were rotated beforehand."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(6)
    grid, H, pairs = (4, 16, 16), 4, (22, 21, 21)
    N = 4 * 16 * 16
    q, k, v = (normal(g, 1, N, H, 128) for _ in range(3))
    freq = bsa.rope_frequencies(pairs)

    def request(q, k):
        mask = bsa.sparsify_topk(q, k, 64, 64, 5)
        nqb, nkb = mask.shape[2:]
        o = torch.empty_like(q)
        plan = bsa.plan(mask, 64, 64, bsa.shapes_of(q, k, v, o), head_offset=[h * nqb * nkb for h in range(H)],
                        stride_b=H * nqb * nkb)
        plan.forward(q, k, v, o)
        torch.cuda.synchronize()
        plan.destroy()
        return o, mask

    rq, rk = bsa.rope(q, k, freq=freq, pairs=pairs, grid=grid)
    o, mask = request(rq, rk)
    pos, _ = orope.grid_positions(N, grid)
    for t, r in ((q, rq), (k, rk)):
        want = torch.from_numpy(orope.rotate(tw.f64(t[0]), pos, freq.cpu().numpy(), pairs, True))
        assert float((r[0].double().cpu() - want).abs().max()) < 2.0 ** -8 * 6
    o2, mask2 = request(rq.clone(), rk.clone())
    assert torch.equal(mask, mask2) and torch.equal(o, o2)
    assert not torch.equal(mask, request(q, k)[1])
