"""Strides of axes of length 1, on the host (no GPU needed).  Made-up addresses: a call that
passes the checks ends at the limit of a launch's threads, before any device work."""
import pytest

from tests.test_ops_host import LIB, UNSUPPORTED, _ffi, backward, forward, grads, window


@pytest.mark.parametrize("token", [1 << 23, 1 << 28, 1 << 40])
def test_token_stride_of_one_token_is_not_looked_at(token):
    one = dict(batch=1 << 27, heads=1, kv_heads=1, seq_q=1, seq_kv=1)
    st = (128, 128, token)
    s = window(q_stride=st, k_stride=st, v_stride=st, o_stride=st, **one)
    g = grads(s, do_stride=st, dq_stride=st, dk_stride=st, dv_stride=st)
    for status in (forward(s), backward(s, g)):
        assert status == _ffi.BSA_ERR_HIP and "configuration" in LIB.bsa_ops_last_error().decode()
    # with a second key it is
    s = window(k_stride=(1 << 41, 128, token), **{**one, "batch": 1, "seq_kv": 2})
    assert forward(s) == UNSUPPORTED and "token stride of k" in LIB.bsa_ops_last_error().decode()
