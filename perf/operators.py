"""Rotary positions and window attention: what a pass over them costs.

Two operators of the package, each in every direction that a program uses:

  rope    rotary positions on up to three axes (time, height, width) of Q and K, the
          inverse rotation that takes their gradients back, and the form that writes the
          rotated keys and the values of new tokens into the rows of a cache
  window  attention over a sliding window and a few first tokens that stay visible:
          prefill, single tokens over a cache, and a training step (forward and backward)

``own`` selects the package's kernels; otherwise the same results are computed from
elementary torch operations in 32 bits (64 for the angles).  Sequences of a batch may
have different lengths; rows behind a sequence's end keep what they held (zeros here).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _rope(name, B, H, Hkv, N, d, dtype, pairs, interleaved, grid=(0, 0, 0), origin=0, inverse=False, cache=0,
          ragged=False, shared=False):
    c = dict(op="rope", B=B, H=H, Hkv=Hkv, N=N, d=d, dtype=dtype, p0=pairs[0], p1=pairs[1], p2=pairs[2],
             interleaved=interleaved, g0=grid[0], g1=grid[1], g2=grid[2], origin=origin, inverse=inverse, cache=cache,
             ragged=ragged, shared=shared)
    if name:
        c["name"] = name
    return c


def _window(name, B, H, Hkv, Nq, Nkv, d, dtype, left, right, sinks, ragged=False, train=False):
    c = dict(op="window", B=B, H=H, Hkv=Hkv, Nq=Nq, Nkv=Nkv, d=d, dtype=dtype, left=left, right=right, sinks=sinks,
             ragged=ragged, train=train)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one new token for each of 16 streams, text and image positions on three axes: the rotated key and the value
        # go into the streams' caches
        _rope("rope_append_token", 16, 32, 8, 1, 128, "bf16", (16, 24, 24), False, cache=1024, shared=True),
        # Q and K of a five-second 720p clip (115200 tokens on a 32 x 45 x 80 grid, 24 heads) before its attention
        _rope("rope_clip_115k", 1, 24, 24, 115200, 128, "bf16", (22, 21, 21), True, grid=(32, 45, 80)),
        # gradients of a training batch in 32 bits: clips of different lengths with unrotated text tokens behind them
        _rope("rope_grad_f32", 2, 12, 12, 5003, 64, "f32", (8, 12, 12), True, grid=(9, 23, 24), origin=3, inverse=True,
              ragged=True),
        # the smallest call: one token of one stream over a 1024-token window
        _window("token_single", 1, 32, 8, 1, 2048, 128, "bf16", 1023, 0, 4, ragged=True),
        # a full serving batch: 64 streams of different lengths, 4096-token window in a 16384-token cache
        _window("token_batch64", 64, 32, 8, 1, 16384, 128, "bf16", 4095, 0, 4, ragged=True),
        # five drafted tokens a stream are looked at together
        _window("token_five_f16", 4, 16, 4, 5, 5000, 64, "f16", 2047, 0, 16, ragged=True),
        # the prompt of one stream
        _window("prefill_16k", 1, 32, 8, 16384, 16384, 128, "bf16", 4095, 0, 4),
        # a small batch of prompts of odd lengths, narrow heads
        _window("prefill_ragged_f16", 3, 16, 16, 5001, 5001, 64, "f16", 700, 0, 1, ragged=True),
        # every frame of the 720p clip sees two frames before and behind it and the first one
        _window("clip_115k", 1, 24, 24, 115200, 115200, 128, "bf16", 7200, 7200, 3600),
        # training steps: a language layer with shared key heads ...
        _window("train_8k", 1, 16, 4, 8192, 8192, 128, "bf16", 1023, 0, 4, train=True),
        # ... a ragged batch of short sequences, window on both sides ...
        _window("train_ragged_f16", 4, 8, 8, 1501, 1501, 64, "f16", 255, 64, 0, ragged=True, train=True),
        # ... and eight frames of a clip, one frame of window on each side and the first one
        _window("train_clip_28k", 1, 24, 24, 28800, 28800, 128, "bf16", 3600, 3600, 3600, train=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("rope", "rope", "token", "token", "prefill", "prefill", "train", "train"))
    dtype = rng.choice(("bf16", "f16"))
    d = rng.choice((64, 128))
    Hkv = rng.choice((1, 2, 3, 4, 8))
    H = Hkv * rng.choice((1, 1, 2, 4, 5, 8))
    sinks = rng.choice((0, 1, 4, 16, _log(rng, 20, 1000)))
    if kind == "rope":
        dtype = rng.choice(("bf16", "f16", "f32"))
        d = rng.choice((64, 72, 96, 128, 256))
        p = d // 2
        a, b = rng.randint(1, p // 2), rng.randint(1, p // 4)
        pairs = rng.choice(((p, 0, 0), (p - a - b, a, b), (p // 2 - b, b, 0)))
        il = rng.choice((True, False))
        how = rng.choice(("grid", "positions", "cache"))
        if how == "cache":
            N = rng.choice((1, 1, 2, 7))
            return _rope("", _log(rng, 1, 64), H, Hkv, N, d, dtype, pairs, il, cache=_log(rng, 16, 512), shared=True)
        if how == "positions":
            return _rope("", rng.randint(1, 3), H, Hkv, _log(rng, 1, 20000), d, dtype, pairs, il,
                         inverse=rng.choice((True, False)), ragged=True, shared=rng.choice((True, False)))
        g = (_log(rng, 1, 20), _log(rng, 2, 40), _log(rng, 2, 60))
        return _rope("", rng.randint(1, 2), H, Hkv, g[0] * g[1] * g[2] + rng.choice((0, 0, 77)), d, dtype, pairs, il,
                     grid=g, origin=rng.choice((0, 5, 1000)), inverse=rng.choice((True, False)))
    if kind == "token":
        B, Nkv = _log(rng, 1, 64), _log(rng, 30, 16000)
        while B * Nkv * Hkv * d > 1 << 29:
            B = max(1, B // 2)
        left = rng.choice((-1, _log(rng, 1, 8000), _log(rng, 100, 8000)))
        return _window("", B, H, Hkv, rng.choice((1, 1, 1, 2, 5, 17)), Nkv, d, dtype, left, 0, sinks,
                       ragged=rng.choice((True, True, False)))
    train = kind == "train"
    N = _log(rng, 50, 6000 if train else 20000)
    right = rng.choice((0, 0, 0, _log(rng, 1, 2000)))
    left = rng.choice((_log(rng, 16, 4096), _log(rng, 128, 4096), -1 if N < 3000 else 1000))
    Nkv = N if train else N + rng.choice((0, 0, 0, _log(rng, 1, 3000)))
    return _window("", rng.randint(1, 3), min(H, 16 * Hkv), Hkv, N, Nkv, d, dtype, left, right, sinks,
                   ragged=rng.choice((True, False)), train=train)


def _lengths(case):
    """(query, key) lengths of a ragged batch: spread from the whole length down to a small part, set by the sizes alone."""
    B = case["B"]
    if case["op"] == "rope":
        return [max(1, case["N"] - (case["N"] * 3 * b) // (4 * B)) for b in range(B)], None
    nq, nkv = case["Nq"], case["Nkv"]
    if nq * 4 <= nkv:  # tokens over a cache: every query row counts, the caches are filled differently
        return [nq] * B, [max(1, nkv - 1 - (nkv * 5 * b) // (6 * B)) for b in range(B)]
    q = [max(1, nq - (nq * 3 * b) // (4 * B)) for b in range(B)]
    return q, [min(nkv, n + nkv - nq) for n in q]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    t = DTYPES[case["dtype"]]
    B, H, Hkv, d = case["B"], case["H"], case["Hkv"], case["d"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32).to(t)

    def ints(v):
        return torch.tensor(v, dtype=torch.int32, device="cuda")

    s = dict(case=case)
    qlen, kvlen = _lengths(case) if case["ragged"] else (None, None)
    if case["op"] == "rope":
        N, cap = case["N"], case["cache"]
        s["q"], s["k"] = normal(B, N, H, d), normal(B, N, Hkv, d)
        s["v"] = normal(B, N, Hkv, d) if cap else None
        s["lengths"] = ints(qlen) if qlen else None
        s["q_out"] = torch.zeros_like(s["q"])
        s["k_out"] = torch.zeros((B, cap, Hkv, d), dtype=t, device="cuda") if cap else torch.zeros_like(s["k"])
        s["v_out"] = torch.zeros_like(s["k_out"]) if cap else None
        s["rows"] = ints([(cap - N) * b // max(1, B) for b in range(B)]) if cap else None
        s["positions"] = None
        if not case["g0"]:
            first = torch.randint(0, 100000, (3, B, 1), generator=g, device="cuda", dtype=torch.int32)
            s["positions"] = (first + torch.arange(N, device="cuda", dtype=torch.int32)).contiguous()
        pairs = [p for p in (case["p0"], case["p1"], case["p2"]) if p]
        # frequency and axis of each rotated pair: theta^(-i/n) over the axis's own pairs, or over all of them
        n_all = sum(pairs)
        freq, axis = [], []
        for a, n in enumerate(pairs):
            for i in range(n):
                freq.append(10000.0 ** (-(len(freq) / n_all if case["shared"] else i / n)))
                axis.append(a)
        s["freq"] = torch.tensor(freq, dtype=torch.float64, device="cuda")
        s["axis"] = torch.tensor(axis, device="cuda")
        s["pairs"] = pairs
        return s
    nq, nkv = case["Nq"], case["Nkv"]
    s["q"], s["k"], s["v"] = normal(B, nq, H, d), normal(B, nkv, Hkv, d), normal(B, nkv, Hkv, d)
    if case["sinks"]:
        # the first tokens draw weight from every query
        n = min(case["sinks"], 4, nkv)
        c = torch.randn((d,), generator=g, device="cuda") * 0.5
        s["k"][:, :n] += c.to(t)
        s["q"] += c.to(t)
    s["q_len"], s["kv_len"] = (ints(qlen), ints(kvlen)) if qlen else (None, None)
    s["o"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros((B, H, nq), dtype=torch.float32, device="cuda")
    if case["train"]:
        s["do"] = normal(B, nq, H, d)
        s["dq"], s["dk"], s["dv"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"]), torch.zeros_like(s["v"])
    return s


def run(s):
    if s["case"]["op"] == "rope":
        return _rope_own(s) if own else _rope_plain(s)
    return _window_own(s) if own else _window_plain(s)


# ----------------------------------------------------------------------------
# The package's kernels

def _rope_own(s):
    import paper_2609_25869_amd as bsa
    c = s["case"]
    bsa.rope(s["q"], s["k"], s["v"], freq=s["freq"], pairs=s["pairs"], interleaved=c["interleaved"],
             positions=s["positions"], grid=(c["g0"], c["g1"], c["g2"]) if c["g0"] else None,
             origin=(c["origin"], 0, 0), lengths=s["lengths"], rows=s["rows"], out_q=s["q_out"], out_k=s["k_out"], out_v=s["v_out"], inverse=c["inverse"])
    return [x for x in (s["q_out"], s["k_out"], s["v_out"]) if x is not None]


def _window_own(s):
    import paper_2609_25869_amd as bsa
    c = s["case"]
    how = dict(q_len=s["q_len"], kv_len=s["kv_len"])
    bsa.window_forward(s["q"], s["k"], s["v"], c["left"], c["right"], c["sinks"], o=s["o"], lse=s["lse"], **how)
    out = {"o": s["o"], "lse": s["lse"]}
    if c["train"]:
        bsa.window_backward(s["q"], s["k"], s["v"], s["o"], s["lse"], s["do"], c["left"], c["right"], c["sinks"],
                            dq=s["dq"], dk=s["dk"], dv=s["dv"], **how)
        out.update(dq=s["dq"], dk=s["dk"], dv=s["dv"])
    return out


# ----------------------------------------------------------------------------
# The plain forms

def _rope_plain(s):
    c = s["case"]
    B, N = c["B"], c["N"]
    n = torch.arange(N, device="cuda")
    if s["positions"] is not None:
        pos, turned = s["positions"].double(), torch.ones(N, dtype=torch.bool, device="cuda")
    else:
        w, hw = c["g2"], c["g1"] * c["g2"]
        pos = torch.stack([n // hw + c["origin"], n // w % c["g1"], n % w]).double()[:, None].expand(3, B, N)
        turned = n < c["g0"] * hw
    angle = torch.remainder(pos[s["axis"]].permute(1, 2, 0) * s["freq"], 2 * math.pi)  # [B, N, pairs]
    angle = torch.where(turned[None, :, None], angle, 0.0)
    co, si = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    si = -si if c["inverse"] else si
    keep = (n < s["lengths"][:, None] if s["lengths"] is not None else n[None].expand(B, N) >= 0)[:, :, None, None]

    def turn(x):
        P = s["freq"].numel()
        a = x.float()
        u, v = (a[..., 0:2 * P:2], a[..., 1:2 * P:2]) if c["interleaved"] else (a[..., :P], a[..., P:2 * P])
        ru, rv = u * co - v * si, u * si + v * co
        r = torch.stack([ru, rv], -1).flatten(-2) if c["interleaved"] else torch.cat([ru, rv], -1)
        return torch.where(keep, torch.cat([r, a[..., 2 * P:]], -1), 0.0).to(x.dtype)

    q, k = turn(s["q"]), turn(s["k"])
    if s["rows"] is None:
        return [q, k]
    at = (s["rows"][:, None] + n).long()
    b = torch.arange(B, device="cuda")[:, None]
    s["k_out"][b, at] = k
    s["v_out"][b, at] = s["v"]
    return [q, s["k_out"], s["v_out"]]


def _window_plain(s):
    """Rows in chunks; each chunk against the keys that any of its rows may see, taken by index."""
    c = s["case"]
    B, H, Hkv, nq, nkv, d = c["B"], c["H"], c["Hkv"], c["Nq"], c["Nkv"], c["d"]
    G, left, right, sinks = H // Hkv, c["left"], c["right"], min(c["sinks"], c["Nkv"])
    scale = 1.0 / math.sqrt(d)
    dev = "cuda"
    qlen = s["q_len"] if s["q_len"] is not None else torch.full((B,), nq, dtype=torch.int32, device=dev)
    kvlen = s["kv_len"] if s["kv_len"] is not None else torch.full((B,), nkv, dtype=torch.int32, device=dev)
    off = (kvlen - qlen).long()
    q = s["q"].float().view(B, nq, Hkv, G, d).permute(0, 2, 1, 3, 4)  # [B, Hkv, Nq, G, d]
    o = torch.zeros((B, Hkv, nq, G, d), device=dev)
    lse = torch.zeros((B, Hkv, nq, G), device=dev)
    train = c["train"]
    if train:
        do = s["do"].float().view(B, nq, Hkv, G, d).permute(0, 2, 1, 3, 4)
        dq = torch.zeros_like(o)
        dk = torch.zeros((B * nkv, Hkv, d), device=dev)
        dv = torch.zeros_like(dk)
    span = nkv if left < 0 else min(nkv, left + right + 1)
    chunk = max(1, min(nq, (1 << 28) // max(1, B * H * (span + sinks))))
    for i0 in range(0, nq, chunk):
        i = torch.arange(i0, min(nq, i0 + chunk), device=dev)
        R = i.numel()
        width = nkv if left < 0 else min(nkv, left + right + R)
        p = i + off[:, None]                                   # [B, R] positions of the rows
        lo = (p - left).clamp(min=0) if left >= 0 else torch.zeros_like(p)
        hi = torch.minimum(p + right, kvlen.long()[:, None] - 1)
        first = lo[:, :1].clamp(max=nkv - width)               # [B, 1]
        j = torch.cat([first + torch.arange(width, device=dev),
                       torch.arange(sinks, device=dev).expand(B, sinks)], 1)  # [B, C]
        jj = j[:, None]                                        # [B, 1, C]
        see = (jj <= hi[:, :, None]) & (i < qlen[:, None])[:, :, None]
        inside = torch.arange(j.shape[1], device=dev) < width
        see = see & torch.where(inside, jj >= lo[:, :, None], jj < lo[:, :, None])
        at = (j + torch.arange(B, device=dev)[:, None] * nkv).flatten()
        kc = s["k"].reshape(B * nkv, Hkv, d)[at].float().view(B, -1, Hkv, d).permute(0, 2, 1, 3).contiguous()
        vc = s["v"].reshape(B * nkv, Hkv, d)[at].float().view(B, -1, Hkv, d).permute(0, 2, 1, 3).contiguous()
        qc = q[:, :, i0:i0 + R].reshape(B, Hkv, R * G, d)
        hide = ~see.repeat_interleave(G, 1)[:, None]           # [B, 1, R * G, C]
        sc = torch.matmul(qc, kc.transpose(2, 3).contiguous()).mul_(scale).masked_fill_(hide, -math.inf)
        m = sc.amax(-1, keepdim=True)
        m = torch.where(m == -math.inf, 0.0, m)
        e = sc.sub_(m).exp_()
        z = e.sum(-1, keepdim=True)
        e /= torch.where(z > 0, z, 1.0)
        oc = torch.matmul(e, vc)
        o[:, :, i0:i0 + R] = oc.view(B, Hkv, R, G, d)
        lse[:, :, i0:i0 + R] = (m + z.log()).view(B, Hkv, R, G)
        if train:
            dc = do[:, :, i0:i0 + R].reshape(B, Hkv, R * G, d) * (i < qlen[:, None]).repeat_interleave(G, 1)[:, None, :, None]
            ds = torch.matmul(dc, vc.transpose(2, 3).contiguous())
            ds.sub_((dc * oc).sum(-1, keepdim=True)).mul_(e).mul_(scale)
            dq[:, :, i0:i0 + R] = torch.matmul(ds, kc).view(B, Hkv, R, G, d)
            back = lambda x: x.permute(0, 2, 1, 3).reshape(-1, Hkv, d)
            dk.index_add_(0, at, back(torch.matmul(ds.transpose(2, 3).contiguous(), qc)))
            dv.index_add_(0, at, back(torch.matmul(e.transpose(2, 3).contiguous(), dc)))
    rows = torch.arange(nq, device=dev) < qlen[:, None]
    lse = torch.where(rows[:, None, :, None], lse, 0.0)
    heads = lambda x: x.permute(0, 2, 1, 3, 4).reshape(B, nq, H, d).to(s["q"].dtype)
    out = {"o": heads(o), "lse": lse.permute(0, 1, 3, 2).reshape(B, H, nq).contiguous()}
    if train:
        out.update(dq=heads(dq), dk=dk.view(B, nkv, Hkv, d).to(s["k"].dtype), dv=dv.view(B, nkv, Hkv, d).to(s["v"].dtype))
    return out


# ----------------------------------------------------------------------------
# What a pass cannot do without

def _visible(case):
    """(visible query-key pairs, keys that some row sees) over the batch, one head."""
    qlen, kvlen = _lengths(case) if case["ragged"] else ([case["Nq"]] * case["B"], [case["Nkv"]] * case["B"])
    pairs = keys = 0
    for a, n in zip(qlen, kvlen):
        p = torch.arange(a, dtype=torch.int64) + (n - a)
        hi = (p + case["right"]).clamp(max=n - 1)
        lo = (p - case["left"]).clamp(min=0) if case["left"] >= 0 else torch.zeros_like(p)
        sink = torch.minimum(torch.minimum(lo, hi + 1), torch.tensor(case["sinks"])).clamp(min=0)
        pairs += int(((hi - lo + 1).clamp(min=0) + sink).sum())
        ok = hi >= lo
        seen = int(hi[ok].max() - lo[ok].min() + 1) if bool(ok.any()) else 0
        keys += min(n, seen + int(sink.max()))
    return pairs, keys


def work(case):
    B, H, Hkv, d = case["B"], case["H"], case["Hkv"], case["d"]
    size = torch.finfo(DTYPES[case["dtype"]]).bits // 8
    if case["op"] == "rope":
        n = sum(_lengths(case)[0]) if case["ragged"] else B * case["N"]
        heads = H + (2 if case["cache"] else 1) * Hkv
        return {"bytes": 2 * n * heads * d * size, "flops": 6 * n * (H + Hkv) * (case["p0"] + case["p1"] + case["p2"])}
    pairs, keys = _visible(case)
    rows = sum(_lengths(case)[0]) if case["ragged"] else B * case["Nq"]
    kv = 2 * keys * Hkv * d * size
    if not case["train"]:
        return {"bytes": kv + rows * H * (2 * d * size + 4), "flops": 4 * d * H * pairs}
    # forward, then backward: q, k, v twice, o and lse written and read, do read, three gradients written
    return {"bytes": 3 * kv + rows * H * (6 * d * size + 8), "flops": 14 * d * H * pairs}


# ----------------------------------------------------------------------------
# The definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    return _rope_exact(case, s) if case["op"] == "rope" else _window_exact(case, s)


def _rope_exact(case, s):
    """Pairs as complex numbers times e^(i angle)."""
    B, N = case["B"], case["N"]
    P = s["freq"].numel()
    outs = []
    for name in ("q", "k"):
        x = s[name]
        full = torch.zeros((B, s["k_out"].shape[1]) + tuple(x.shape[2:]) if name == "k" else tuple(x.shape),
                           dtype=torch.float64, device="cuda")
        for b in range(B):
            n = torch.arange(N, device="cuda")
            if s["positions"] is not None:
                at = s["positions"][:, b].double()
            else:
                t, r = n // (case["g1"] * case["g2"]), n % (case["g1"] * case["g2"])
                at = torch.stack([t + case["origin"], r // case["g2"], r % case["g2"]]).double()
                at = at * (n < case["g0"] * case["g1"] * case["g2"])
                if case["origin"]:
                    at[0] = torch.where(n < case["g0"] * case["g1"] * case["g2"], at[0], 0.0)
            theta = at[s["axis"]].T * s["freq"]
            z = torch.polar(torch.ones_like(theta), -theta if case["inverse"] else theta)[:, None]
            a = x[b].double()
            r = a.clone()
            if case["interleaved"]:
                y = torch.complex(a[..., 0:2 * P:2].contiguous(), a[..., 1:2 * P:2].contiguous()) * z
                r[..., 0:2 * P:2], r[..., 1:2 * P:2] = y.real, y.imag
            else:
                y = torch.complex(a[..., :P].contiguous(), a[..., P:2 * P].contiguous()) * z
                r[..., :P], r[..., P:2 * P] = y.real, y.imag
            row = int(s["rows"][b]) if s["rows"] is not None and name == "k" else 0
            count = int(s["lengths"][b]) if s["lengths"] is not None else N
            full[b, row:row + count] = r[:count]
        outs.append(full)
    if s["v"] is not None:
        full = torch.zeros(tuple(s["v_out"].shape), dtype=torch.float64, device="cuda")
        for b in range(B):
            full[b, int(s["rows"][b]):int(s["rows"][b]) + N] = s["v"][b].double()
        outs.append(full)
    return outs


def _window_exact(case, s):
    """Dense scores of one sequence and head at a time under a dense mask."""
    B, H, Hkv, d = case["B"], case["H"], case["Hkv"], case["d"]
    nq, nkv = case["Nq"], case["Nkv"]
    if B * H * nq * nkv > 2.5e10:
        return None
    o = torch.zeros((B, nq, H, d), dtype=torch.float64, device="cuda")
    lse = torch.zeros((B, H, nq), dtype=torch.float64, device="cuda")
    if case["train"]:
        dq, dk, dv = (torch.zeros(tuple(s[n].shape), dtype=torch.float64, device="cuda") for n in ("q", "k", "v"))
    for b in range(B):
        a = int(s["q_len"][b]) if s["q_len"] is not None else nq
        n = int(s["kv_len"][b]) if s["kv_len"] is not None else nkv
        for r0 in range(0, a, 8192):
            r1 = min(a, r0 + 8192)
            i = torch.arange(r0, r1, device="cuda")[:, None] + (n - a)
            j = torch.arange(n, device="cuda")[None]
            ok = j <= i + case["right"]
            if case["left"] >= 0:
                ok &= (j >= i - case["left"]) | (j < case["sinks"])
            for h in range(H):
                kv = h // (H // Hkv)
                q, k, v = s["q"][b, r0:r1, h].double(), s["k"][b, :n, kv].double(), s["v"][b, :n, kv].double()
                score = torch.where(ok, q @ k.T / d ** 0.5, -math.inf)
                l = torch.logsumexp(score, 1)
                lse[b, h, r0:r1] = l
                p = torch.where(ok, torch.exp(score - torch.where(l == -math.inf, 0.0, l)[:, None]), 0.0)
                del score
                out = p @ v
                o[b, r0:r1, h] = out
                if case["train"]:
                    g = s["do"][b, r0:r1, h].double()
                    dv[b, :n, kv] += p.T @ g
                    ds = p * (g @ v.T - (g * out).sum(1)[:, None]) / d ** 0.5
                    dq[b, r0:r1, h] = ds @ k
                    dk[b, :n, kv] += ds.T @ q
                    del ds
                del p
    out = {"o": o, "lse": lse}
    if case["train"]:
        out.update(dq=dq, dk=dk, dv=dv)
    return out
