"""Calls of the operators that torch would record: they say that they carry no gradients."""
import warnings

import pytest

pytestmark = pytest.mark.gpu

import paper_2609_25869_amd as bsa  # noqa: E402  (fails loudly if the libraries are missing)


def test_calls_that_are_not_recorded_say_so():
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = [torch.randn((1, 9, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(3)]
    freq = bsa.rope_frequencies((32,))
    pos = torch.arange(9, dtype=torch.int32, device="cuda").view(1, 1, 9)
    calls = {"window_forward": lambda q, k, v: bsa.window_forward(q, k, v, 3),
             "rope": lambda q, k, v: bsa.rope(q, k, v, freq=freq, pairs=(32,), positions=pos)}
    for name, call in calls.items():
        want = call(*x)
        for i in range(3):
            y = [t.clone().requires_grad_() if i == j else t for j, t in enumerate(x)]
            with pytest.warns(UserWarning, match=name + " takes no part in autograd") as seen:
                got = call(*y)
            assert seen[0].filename == __file__
            assert all(torch.equal(a, b) and not b.requires_grad for a, b in zip(want, got))
            # nothing is lost where nothing is recorded
            with warnings.catch_warnings():
                warnings.simplefilter("error")
                with torch.no_grad():
                    call(*y)
                call(*x)
                call(*(t.detach() for t in y))


def test_operators_within_an_autograd_function():
    """The way into autograd: forward and backward of a user's own function."""
    import torch

    class Window(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v):
            o, lse = bsa.window_forward(q, k, v, 4, 0, 1)
            ctx.save_for_backward(q, k, v, o, lse)
            return o

        @staticmethod
        def backward(ctx, do):
            return bsa.window_backward(*ctx.saved_tensors, do.contiguous(), 4, 0, 1)

    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    q, k, v, do = (torch.randn((2, 30, 2, 64), generator=g, device="cuda").bfloat16() for _ in range(4))
    leaves = [t.clone().requires_grad_() for t in (q, k, v)]
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        Window.apply(*leaves).backward(do)
        o, lse = bsa.window_forward(q, k, v, 4, 0, 1)
        want = bsa.window_backward(q, k, v, o, lse, do, 4, 0, 1)
    torch.cuda.synchronize()
    assert all(torch.equal(a.grad, b) for a, b in zip(leaves, want))
