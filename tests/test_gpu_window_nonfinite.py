"""Values of V that are not finite, on the device: what reaches the queries that see
them, where their weight leaves 32 bits, and what that costs."""
import numpy as np
import pytest

from oracle import window as owin
from tests.gpu_util import log
from tests.test_gpu_window import CASES, F, SENTINEL, STEP, U, close, f64, make, sentinels

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


# name: B, H, Hkv, Nq, Nkv, d, left, right, sinks, q_len, kv_len
SEEN = {
    "token": (2, 4, 2, 1, 90, 128, 40, 0, 2, None, [90, 33]),
    "token_slices": (2, 6, 3, 1, 2500, 64, 2000, 0, 40, None, [2500, 700]),
    "token_slices_128": (1, 8, 2, 3, 3001, 128, -1, 0, 0, None, None),
    "prompt_64": (2, 4, 2, 333, 333, 64, 50, 7, 3, [333, 200], [333, 200]),
    "prompt_128": (2, 4, 2, 333, 333, 128, 50, 7, 3, [333, 200], [333, 200]),
    "prompt_slices": (1, 2, 1, 130, 1500, 128, -1, 0, 0, None, None),
    "prompt_slices_64": (1, 2, 1, 130, 1500, 64, 1400, 0, 5, None, None),
}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("case", list(SEEN))
def test_each_query_gets_what_it_sees(case, dtype, monkeypatch):
    """Infinities of both signs and NaN in single elements of V, in the first key, the last one
    and some between: a column is the sum of the weights (all above 0) times what its query
    sees; the other columns and queries are as without."""
    import torch
    monkeypatch.setitem(CASES, case, SEEN[case])
    x, lens, win, clipped = make(case, dtype, seed=21)
    B, Nkv, Hkv, d = x["v"].shape
    Nq, H = x["q"].shape[1:3]
    kv = clipped["kv_len"] or [Nkv] * B
    rng = np.random.default_rng(22)
    bad = np.zeros((B, Nkv, Hkv, d))
    for b in range(B):
        for j in {0, kv[b] - 1, kv[b] // 2, kv[b] // 2 + 1, *rng.integers(0, kv[b], 4).tolist()}:
            for h in range(Hkv):
                for value, c in zip((INF, -INF, NAN, INF, -INF), rng.integers(0, d - 8, 5)):
                    bad[b, j, h, c] = value
        bad[b, 0, :, 1], bad[b, kv[b] - 1, :, 1] = INF, -INF  # NaN for those that see both
        bad[b, kv[b] - 1, 0, d - 8:] = INF
    mark = torch.from_numpy(bad).cuda()
    x["v"] = torch.where(mark == 0, x["v"], 0)
    r = owin.window_attention(*(f64(x[n]) for n in "qkv"), *win, **clipped)
    x["v"] = torch.where(mark == 0, x["v"], mark.to(x["v"].dtype))
    want = r["o"].copy()
    with np.errstate(invalid="ignore"):
        for b in range(B):
            ql = clipped["q_len"][b] if clipped["q_len"] else Nq
            sees = owin.mask_of(ql, kv[b], ql, kv[b], *win)
            for j, h, c in np.argwhere(bad[b] != 0):
                rows = np.nonzero(sees[:, j])[0]
                for q in range(h * H // Hkv, (h + 1) * H // Hkv):
                    want[b, rows, q, c] += bad[b, j, h, c]
    o, lse, *_ = sentinels(x)
    bsa.window_forward(x["q"], x["k"], x["v"], *win, o=o, lse=lse, **lens)
    torch.cuda.synchronize()
    got, e = f64(o), r["err"]
    none = np.isnan(r["o"])
    assert np.all(got[none] == SENTINEL) and not np.isfinite(want[~none]).all() and np.isfinite(want[~none]).any()
    tol = 1.01 * U[dtype] * (e["o_u"] + np.abs(r["o"])) + STEP[dtype] * e["o_s"] + F * e["o_u"]
    with np.errstate(invalid="ignore"):
        ok = np.where(np.isfinite(want), np.abs(got - want) <= tol, (got == want) | (np.isnan(got) & np.isnan(want)))
    assert ok[~none].all(), np.argwhere(~ok & ~none)[0]
    close("lse", lse, r["lse"], F)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("every", [False, True])
def test_rows_that_are_formed_again_cost_a_walk(d, every):
    """One infinity that all queries see, or one in every value: the rows are walked once more
    with matrix instructions.  (A walk key by key took 130 to 200 times the call here.)"""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    q, k, v = (torch.randn((1, 2048, 8, d), generator=g, device="cuda").bfloat16() for _ in range(3))

    def us():
        times = []
        for _ in range(7):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            bsa.window_forward(q, k, v, -1)
            b.record()
            b.synchronize()
            times.append(1e3 * a.elapsed_time(b))
        return sorted(times)[3]

    us()
    plain = us()
    if every:
        v[..., 3] = INF
    else:
        v[0, 0, :, 3] = INF
    again = us()
    log("d %d %s: %.0f us, with infinities %.0f us" % (d, "every value" if every else "one value", plain, again))
    assert again < 20 * plain
