"""Window attention on the device against the fp64 oracle.

Tolerances count roundings.  A value rounded to T is off by u = eps(T) / 2 of
itself at most; float16 probabilities and score gradients below 2^-14 by 2^-25
instead.  The oracle returns the sums that carry those errors to an output.
32-bit arithmetic: the scores here sum at most 128 products of |q k| < 1 on
average, so they are off by less than 128 * 2^-24 * 128 / sqrt(128) < 1e-4, as
are a row's sum and its LSE; F covers numerator and sum, and twice that where
the backward pass adds the LSE's own error.
"""
import numpy as np
import pytest

from oracle import window as owin
from tests.gpu_util import log

pytestmark = pytest.mark.gpu

import paper_2609_25869_amd as bsa  # noqa: E402  (fails loudly if the libraries are missing)

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11}
STEP = {"bf16": 0.0, "f16": 2.0 ** -25}
F = 2e-4
SENTINEL = 7.25

# name: B, H, Hkv, Nq, Nkv, d, left, right, sinks, q_len, kv_len
CASES = {
    "one_token_one_key": (1, 1, 1, 1, 1, 128, 0, 0, 0, None, None),
    "one_token_cache": (2, 8, 2, 1, 300, 128, 63, 0, 4, None, [300, 117]),
    "one_token_all_keys": (1, 4, 1, 1, 1000, 64, -1, 0, 0, None, None),
    "one_token_long_split": (2, 6, 3, 1, 2500, 128, 2000, 0, 40, None, [2500, 3]),
    "drafted": (3, 8, 2, 5, 700, 64, 129, 0, 2, [5, 3, 0], [700, 64, 10]),
    "rows_33": (1, 33, 1, 1, 500, 128, -1, 0, 0, None, None),
    "square_causal": (1, 2, 2, 257, 257, 128, -1, 0, 0, None, None),
    "square_window": (2, 4, 2, 301, 301, 128, 50, 0, 3, None, None),
    "window_zero": (1, 2, 1, 70, 70, 64, 0, 0, 0, None, None),
    "both_sides": (1, 3, 3, 333, 333, 128, 40, 25, 0, None, None),
    "full": (1, 2, 1, 130, 190, 64, -1, -1, 0, None, None),
    "right_only": (1, 2, 2, 100, 100, 128, 0, -1, 0, None, None),
    "sinks_wide": (1, 2, 1, 400, 400, 128, 30, 0, 100, None, None),
    "sinks_past_keys": (1, 2, 1, 40, 40, 64, 3, 0, 1000, None, None),
    "sinks_touch_tile": (1, 1, 1, 300, 300, 128, 64, 0, 32, None, None),
    "more_queries_than_keys": (2, 4, 2, 90, 33, 128, 20, 0, 2, None, [33, 0]),
    "more_queries_right": (1, 2, 2, 50, 20, 64, 5, 10, 1, None, None),
    "ragged": (4, 6, 2, 200, 260, 128, 60, 7, 5, [200, 1, 0, 77], [260, 1, 50, 40]),
    "ragged_f": (3, 5, 1, 150, 150, 64, 33, 0, 1, [150, 149, 2], [150, 149, 2]),
    "group_7": (1, 7, 1, 65, 65, 64, 31, 0, 0, None, None),
    "group_16": (1, 16, 1, 40, 140, 128, 70, 3, 6, None, None),
    # enough rows for the kernel of 256-row tiles
    "many_rows": (4, 64, 64, 300, 300, 128, 90, 0, 5, None, None),
    "many_rows_shared": (8, 64, 32, 170, 210, 64, 45, 20, 33, [170, 1, 0, 99, 170, 30, 128, 129],
                         [210, 1, 50, 60, 210, 200, 128, 170]),
    "many_rows_group_16": (16, 256, 16, 30, 130, 128, 64, 0, 1, None, None),
    "many_rows_all_keys": (2, 128, 128, 257, 257, 64, -1, 0, 0, None, None),
    "no_keys": (2, 2, 1, 5, 0, 64, 4, 0, 1, None, None),
    "no_queries": (1, 2, 1, 0, 20, 64, 4, 0, 1, None, None),
    "lengths_out_of_range": (3, 2, 1, 20, 30, 64, 6, 0, 1, [25, -3, 20], [99, 30, -1]),
}


def make(case, dtype, seed=0, dv=None):
    import torch
    B, H, Hkv, Nq, Nkv, d, left, right, sinks, ql, kl = CASES[case]
    g = torch.Generator(device="cuda")
    g.manual_seed(1000 + seed)
    t = {"bf16": torch.bfloat16, "f16": torch.float16}[dtype]
    n = lambda *s: torch.randn(s, generator=g, device="cuda").to(t)
    x = dict(q=n(B, Nq, H, d), k=n(B, Nkv, Hkv, d), v=n(B, Nkv, Hkv, d), do=n(B, Nq, H, d))
    lens = dict(q_len=None if ql is None else torch.tensor(ql, dtype=torch.int32, device="cuda"),
                kv_len=None if kl is None else torch.tensor(kl, dtype=torch.int32, device="cuda"))
    clip = lambda l, most: None if l is None else [min(max(a, 0), most) for a in l]
    return x, lens, (left, right, sinks), dict(q_len=clip(ql, Nq), kv_len=clip(kl, Nkv))


def f64(t):
    return t.detach().double().cpu().numpy()


def expect(x, win, lens, **kw):
    return owin.window_attention(f64(x["q"]), f64(x["k"]), f64(x["v"]), *win, do=f64(x["do"]), **lens, **kw)


def close(name, got, ref, tol):
    """Rows that the oracle leaves NaN must hold the sentinel."""
    got = f64(got)
    rows = np.isnan(ref)
    assert np.all(got[rows] == SENTINEL), "%s: rows behind a sequence were written" % name
    bad = ~rows & ~((np.abs(got - ref) <= tol) | (np.isinf(ref) & (got == ref)))
    worst = np.nanmax(np.where(rows | np.isinf(ref), 0, np.abs(got - ref) / np.maximum(tol, 1e-30)), initial=0)
    assert not bad.any(), "%s: %d values off, worst %.3g of the tolerance at %s" % (
        name, bad.sum(), worst, np.argwhere(bad)[0])
    return worst


def check_forward(o, lse, r, dtype, what):
    u, st, e = U[dtype], STEP[dtype], r["err"]
    a = close(what + " o", o, r["o"], 1.01 * u * (e["o_u"] + np.abs(r["o"])) + st * e["o_s"] + F * e["o_u"])
    b = close(what + " lse", lse, r["lse"], F)
    return a, b


def check_backward(dq, dk, dv, r, dtype, what):
    u, st, e = U[dtype], STEP[dtype], r["err"]
    worst = []
    for n, t in (("dq", dq), ("dk", dk)):
        tol = 1.01 * u * (e[n + "_u"] + np.abs(r[n])) + st * e[n + "_s"] + 2 * F * e[n + "_f"] + st
        worst.append(close(what + " " + n, t, r[n], tol))
    tol = 1.01 * u * (e["dv_u"] + np.abs(r["dv"])) + st * e["dv_s"] + 2 * F * e["dv_u"] + st
    worst.append(close(what + " dv", dv, r["dv"], tol))
    return worst


def sentinels(x):
    import torch
    f = lambda t: torch.full_like(t, SENTINEL)
    B, Nq, H, _ = x["q"].shape
    return f(x["q"]), torch.full((B, H, Nq), SENTINEL, device="cuda"), f(x["q"]), f(x["k"]), f(x["v"])


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", list(CASES))
def test_forward_and_backward(case, dtype):
    import torch
    x, lens, win, clipped = make(case, dtype)
    r = expect(x, win, clipped)
    o, lse, dq, dk, dv = sentinels(x)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse, **lens)
    torch.cuda.synchronize()
    a = check_forward(o, lse, r, dtype, case)
    bsa.window_backward(x["q"], x["k"], x["v"], o, lse, x["do"], *win, dq=dq, dk=dk, dv=dv, **lens)
    torch.cuda.synchronize()
    b = check_backward(dq, dk, dv, r, dtype, case)
    log("%s %s: of the tolerance o %.2f lse %.2f dq %.2f dk %.2f dv %.2f" % ((case, dtype) + a + tuple(b)))


@pytest.mark.parametrize("case", ["square_window", "one_token_long_split", "ragged"])
def test_scale(case):
    import torch
    x, lens, win, clipped = make(case, "bf16", seed=5)
    r = expect(x, win, clipped, scale=0.02)
    o, lse, dq, dk, dv = sentinels(x)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, scale=0.02, o=o, lse=lse, **lens)
    bsa.window_backward(x["q"], x["k"], x["v"], o, lse, x["do"], *win, scale=0.02, dq=dq, dk=dk, dv=dv, **lens)
    torch.cuda.synchronize()
    check_forward(o, lse, r, "bf16", case)
    check_backward(dq, dk, dv, r, "bf16", case)


@pytest.mark.parametrize("case", ["one_token_cache", "one_token_long_split", "ragged", "square_window", "sinks_wide"])
def test_unseen_memory_does_not_matter(case):
    """NaN and infinity in keys and values that no query sees, and in the rows
    behind a sequence's end."""
    import torch
    x, lens, win, clipped = make(case, "bf16", seed=1)
    B, Nq = x["q"].shape[:2]
    Nkv = x["k"].shape[1]
    if case == "square_window":
        x["q"], x["do"] = x["q"][:, 200:].contiguous(), x["do"][:, 200:].contiguous()  # the last queries alone
        Nq = x["q"].shape[1]
    for b in range(B):
        ql = clipped["q_len"][b] if clipped["q_len"] else Nq
        kl = clipped["kv_len"][b] if clipped["kv_len"] else Nkv
        unseen = ~owin.mask_of(ql, Nkv, ql, kl, *win).any(0)
        for t, bad in (("k", float("nan")), ("v", float("inf"))):
            x[t][b, torch.from_numpy(unseen).cuda()] = bad
        x["q"][b, ql:] = float("nan")
        x["do"][b, ql:] = float("nan")
    r = expect(x, win, clipped)
    o, lse, dq, dk, dv = sentinels(x)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse, **lens)
    torch.cuda.synchronize()
    check_forward(o, lse, r, "bf16", case)
    bsa.window_backward(x["q"], x["k"], x["v"], o, lse, x["do"], *win, dq=dq, dk=dk, dv=dv, **lens)
    torch.cuda.synchronize()
    check_backward(dq, dk, dv, r, "bf16", case)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", ["square_window", "both_sides", "drafted", "ragged_f", "sinks_wide", "one_token_long_split",
                                  "many_rows_all_keys"])
def test_keys_that_are_not_finite_stay_with_their_queries(case, dtype):
    """NaN in a key and infinities in a value: queries that do not see them get what
    they get without, those that do get no number."""
    import torch
    x, lens, win, clipped = make(case, dtype, seed=8)
    B, Nq = x["q"].shape[:2]
    Nkv, Hkv = x["k"].shape[1:3]
    kv = [clipped["kv_len"][b] if clipped["kv_len"] else Nkv for b in range(B)]
    bad = [sorted({n // 2, n // 2 + 3, max(n - 40, 0)}) for n in kv]
    clean = {n: t.clone() for n, t in x.items()}
    for b in range(B):
        for i, j in enumerate(j for j in bad[b] if j < kv[b]):
            for t in (x, clean):
                t["k"][b, j] *= 0.5
            if i == 0:
                x["k"][b, j, :, 5] = float("nan")
            elif i == 1:
                x["v"][b, j, :, 7] = float("inf")
            else:
                x["v"][b, j] = -float("inf")
    r = expect(clean, win, clipped)
    o, lse, *_ = sentinels(x)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse, **lens)
    torch.cuda.synchronize()
    got, u, st, e = f64(o), U[dtype], STEP[dtype], r["err"]
    hit = 0
    for b in range(B):
        ql = clipped["q_len"][b] if clipped["q_len"] else Nq
        sees = owin.mask_of(ql, kv[b], ql, kv[b], *win)[:, [j for j in bad[b] if j < kv[b]]].any(1)
        free = np.nonzero(~sees)[0]
        tol = (1.01 * u * (e["o_u"] + np.abs(r["o"])) + st * e["o_s"] + F * e["o_u"])[b, free]
        assert np.all(np.abs(got[b, free] - r["o"][b, free]) <= tol), "query that sees no such key"
        assert not np.isfinite(got[b, :ql][sees]).all(-1).any(), "query that sees one"
        hit += int(sees.sum())
    assert hit > 0


@pytest.mark.parametrize("layout", ["bhnd", "qkv", "broadcast", "odd_strides"])
def test_strides(layout):
    import torch
    x, lens, win, clipped = make("ragged", "bf16", seed=2)
    B, Nq, H, d = x["q"].shape
    Nkv, Hkv = x["k"].shape[1:3]
    swap = lambda t: t.transpose(1, 2).contiguous().transpose(1, 2)
    if layout == "bhnd":
        x = {n: swap(t) for n, t in x.items()}
    elif layout == "qkv":  # K and V as slices of one buffer
        buf = torch.full((B, Nkv, 3 * Hkv, d), float("nan"), dtype=torch.bfloat16, device="cuda")
        for i, n in enumerate("kv"):
            buf[:, :, i * Hkv:(i + 1) * Hkv] = x[n]
            x[n] = buf[:, :, i * Hkv:(i + 1) * Hkv]
    elif layout == "broadcast":  # one K and V for the batch
        x["k"], x["v"] = x["k"][:1].expand_as(x["k"]), x["v"][:1].expand_as(x["v"])
    else:
        for n in x:
            b, s, h, _ = x[n].shape
            buf = torch.full((b, s + 3, h + 1, d + 8), float("nan"), dtype=torch.bfloat16, device="cuda")
            buf[:, 1:s + 1, :h, :d] = x[n]
            x[n] = buf[:, 1:s + 1, :h, :d]
    r = expect(x, win, clipped)
    o, lse, dq, dk, dv = sentinels({n: t.contiguous() for n, t in x.items()})
    if layout != "broadcast":
        o, dq, dk, dv = swap(o), swap(dq), swap(dk), swap(dv)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse, **lens)
    bsa.window_backward(x["q"], x["k"], x["v"], o, lse, x["do"], *win, dq=dq, dk=dk, dv=dv, **lens)
    torch.cuda.synchronize()
    check_forward(o, lse, r, "bf16", layout)
    check_backward(dq, dk, dv, r, "bf16", layout)


def test_large_scores():
    """Scores of hundreds, rising along the keys: the softmax reference moves."""
    import torch
    x, lens, win, clipped = make("square_causal", "bf16", seed=3)
    ramp = torch.linspace(-3, 3, x["k"].shape[1], device="cuda")[None, :, None, None]
    x["q"] = (x["q"].float() * 0.1 + 2).to(torch.bfloat16)
    x["k"] = (x["k"].float() * 0.1 + 4 * ramp).to(torch.bfloat16)
    r = expect(x, win, clipped)
    o, lse, *_ = sentinels(x)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse)
    torch.cuda.synchronize()
    # scores sum 128 products of up to 24: off by 128 * 2^-24 * 128 * 24 / sqrt(128) < 2.1e-3 at most
    e = r["err"]
    close("o", o, r["o"], 1.01 * U["bf16"] * (e["o_u"] + np.abs(r["o"])) + 5e-3 * e["o_u"])
    close("lse", lse, r["lse"], 5e-3)


def test_far_rows_of_a_long_cache():
    """Byte offsets past 2^32 inside one head's keys."""
    import torch
    n, heads, d = 1100000, 16, 128   # 4096 bytes a token: 4.5 GB
    buf = torch.zeros((1, n, heads, d), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(9)
    tail = torch.randn((1, 400, 2, d), generator=g, device="cuda").to(torch.bfloat16)
    head = torch.randn((1, 8, 2, d), generator=g, device="cuda").to(torch.bfloat16)
    buf[:, -400:, 14:] = tail
    buf[:, :8, 14:] = head
    k, v = buf[:, :, 14:15], buf[:, :, 15:16]
    q = torch.randn((1, 70, 2, d), generator=g, device="cuda").to(torch.bfloat16)
    for nq in (1, 70):
        o, lse = bsa.window_forward(q[:, :nq].contiguous(), k, v, 299, 0, 8)
        torch.cuda.synchronize()
        # the same keys side by side: 8 sinks, then the last 400
        kk = torch.cat([head[:, :, :1], tail[:, :, :1]], 1)
        vv = torch.cat([head[:, :, 1:], tail[:, :, 1:]], 1)
        r = owin.window_attention(f64(q[:, :nq]), f64(kk), f64(vv), 299, 0, 8)
        check_forward(o, lse, r, "bf16", "far %d" % nq)
    del buf, k, v
    torch.cuda.empty_cache()


@pytest.mark.parametrize("case", ["ragged", "one_token_long_split", "sinks_wide"])
def test_same_bits_every_time(case):
    import torch
    x, lens, win, _ = make(case, "bf16", seed=4)

    def once():
        o, lse = bsa.window_forward(x["q"], x["k"], x["v"], *win, **lens)
        return (o, lse) + bsa.window_backward(x["q"], x["k"], x["v"], o, lse, x["do"], *win, **lens)

    first = once()
    for _ in range(3):
        for a, b in zip(first, once()):
            assert torch.equal(a, b)


def test_other_stream_and_own_workspace():
    import torch
    x, lens, win, clipped = make("one_token_long_split", "bf16", seed=6)
    r = expect(x, win, clipped)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    n = bsa.window_workspace(x["q"], x["k"], x["v"], *win)
    nb = bsa.window_workspace(x["q"], x["k"], x["v"], *win, backward=True)
    assert n > 0 and nb > 0
    ws = torch.full((max(n, nb),), 255, dtype=torch.uint8, device="cuda")
    o, lse, dq, dk, dv = sentinels(x)
    torch.cuda.synchronize()
    for handle in (side, side.cuda_stream):
        bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse, workspace=ws, stream=handle, **lens)
        bsa.window_backward(x["q"], x["k"], x["v"], o, lse, x["do"], *win, dq=dq, dk=dk, dv=dv, workspace=ws,
                            stream=handle, **lens)
        side.synchronize()
        check_forward(o, lse, r, "bf16", "side stream")
        check_backward(dq, dk, dv, r, "bf16", "side stream")
    o2, lse2 = bsa.window_forward(x["q"], x["k"], x["v"], *win, stream=side, **lens)
    side.synchronize()
    assert torch.equal(o2, o) and torch.equal(lse2, lse)


def test_captured_and_replayed():
    """Two graphs with workspaces of their own, replayed with new inputs and eager
    work in between."""
    import torch
    cases = ["one_token_long_split", "ragged"]
    made, graphs, outs = [], [], []
    for c in cases:
        x, lens, win, _ = make(c, "bf16", seed=7)
        call = lambda x=x, lens=lens, win=win: (lambda f: f + bsa.window_backward(
            x["q"], x["k"], x["v"], f[0], f[1], x["do"], *win, **lens))(
                bsa.window_forward(x["q"], x["k"], x["v"], *win, **lens))
        call()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = call()
        made.append((x, call))
        graphs.append(g)
        outs.append(out)
    for rep in range(3):
        for (x, call), g, out in zip(made, graphs, outs):
            for t in x.values():
                t.copy_(torch.randn(t.shape, device="cuda").to(t.dtype))
            eager = [t.clone() for t in call()]
            for g2 in graphs:
                g2.replay()
            torch.cuda.synchronize()
            for a, b in zip(eager, out):
                assert torch.equal(a, b), rep
