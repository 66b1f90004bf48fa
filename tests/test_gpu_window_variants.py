"""Window attention's backward kernels one by one: calls of every dK/dV variant with shared
key heads, ragged lengths, both sides of a window and sinks.  test_window_plan_host.py holds
each call to its variant."""
import pytest

from tests import test_gpu_window as tw

pytestmark = pytest.mark.gpu

import paper_2609_25869_amd as bsa  # noqa: E402,F401  (fails loudly if the libraries are missing)

# name: ((B, H, Hkv, Nq, Nkv, d, left, right, sinks, q_len, kv_len), what the plan says)
VARIANTS = {
    # one workgroup per key tile, head dim 128
    "plain": ((4, 96, 48, 300, 300, 128, 90, 20, 0, [300, 1, 0, 170], [300, 200, 50, 171]), dict(deep=0, slices=1)),
    "plain_left": ((6, 90, 30, 290, 290, 128, -1, 0, 0, [290, 289, 129, 128, 3, 64], [290, 290, 129, 128, 200, 65]),
                   dict(deep=0, slices=1)),
    "plain_right": ((6, 60, 30, 290, 290, 128, 0, -1, 0, None, [290, 1, 0, 129, 128, 257]), dict(deep=0, slices=1)),
    "plain_sinks": ((5, 56, 28, 400, 400, 128, 30, 10, 140, [400, 399, 7, 130, 257], [400, 400, 300, 130, 257]),
                    dict(deep=0, slices=1, sink_slices=4)),
    "plain_few_queries": ((3, 120, 30, 100, 700, 128, 150, 5, 3, [100, 65, 1], [700, 640, 129]), dict(deep=0, slices=1)),
    # tiles with and without sinks in slices
    "plain_slices": ((1, 256, 64, 600, 600, 128, 60, 0, 400, [590], [600]), dict(deep=0, slices=3, sink_slices=10)),
    # one wave per SIMD
    "deep": ((2, 12, 4, 333, 333, 128, 70, 30, 0, [333, 130], [333, 131]), dict(deep=1, slices=3)),
    "deep_sinks": ((2, 8, 2, 500, 500, 128, 60, 0, 150, [500, 77], [500, 300]), dict(deep=1, slices=3, sink_slices=8)),
    "deep_whole": ((4, 60, 60, 200, 200, 128, 40, 3, 0, [200, 64, 129, 1], [200, 200, 128, 70]), dict(deep=1, slices=1)),
    # head dim 64
    "d64": ((8, 128, 32, 230, 230, 64, 60, 9, 0, [230, 1, 0, 64, 65, 128, 129, 200], [230, 30, 40, 64, 70, 200, 129, 201]),
            dict(deep=0, slices=1)),
    "d64_slices": ((2, 12, 4, 333, 700, 64, 200, 30, 130, [333, 130], [700, 131]), dict(deep=0, slices=5, sink_slices=5)),
}


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("name", list(VARIANTS))
def test_variant(name, dtype, monkeypatch):
    monkeypatch.setitem(tw.CASES, name, VARIANTS[name][0])
    tw.test_forward_and_backward(name, dtype)


@pytest.mark.parametrize("name", ["plain", "plain_sinks", "plain_few_queries", "plain_slices", "deep", "d64", "d64_slices"])
def test_unseen_memory(name, monkeypatch):
    """NaN in padded query rows and in unseen keys, infinity in unseen values."""
    monkeypatch.setitem(tw.CASES, name, VARIANTS[name][0])
    tw.test_unseen_memory_does_not_matter(name)
