"""Ends of the ranges that the gradient and token calls accept, on the host: no GPU is needed and no pointer
is followed."""
import ctypes
import subprocess
import sys

import pytest

from paper_1508_06904_amd import dss

OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 2, 3
MAX_K = 131071                     # channels whose products of codes stay in 32 bits


@pytest.mark.parametrize("M,N,K", [(40, 8, 2 ** 31 - 1), (2 ** 40, 8, 2 ** 24), (4, 8, MAX_K + 1), (1, 1, 2 ** 31 - 127)])
def test_workspace_query_refuses_sums_over_32_bits(M, N, K):
    """In a process of its own: a division by an overflowed row length would end it."""
    code = ("import ctypes; from paper_1508_06904_amd import dss; n = ctypes.c_int64(-5)\n"
            "for s in range(3): print(dss.lib().dss_tokens_workspace(%d, %d, %d, s, ctypes.byref(n)), n.value)" % (M, N, K))
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.returncode
    assert r.stdout.split() == [str(UNSUPPORTED), "-5"] * 3


@pytest.mark.parametrize("source", [0, 1, 2])
def test_workspace_of_the_largest_layer(source):
    """The largest tokens, outputs and channels together: the bytes fit 64 bits."""
    need = ctypes.c_int64()
    assert dss.lib().dss_tokens_workspace(2 ** 40, 2 ** 20, MAX_K, source, ctypes.byref(need)) == OK
    weights = 2 ** 20 * (MAX_K + 1)
    assert need.value >= weights and need.value >= (2 ** 40 * (MAX_K + 1) if source != 2 else 0)


def test_a_norm_between_words_is_refused():
    VP, at = ctypes.c_void_p, 1 << 20
    for off in (1, 2, 3):
        assert dss.lib().dss_grad_norm(None, 0, VP(at + off), VP(at), 8192, None) == INVALID
        assert dss.lib().dss_clip_grads(None, None, 0, 1.0, VP(at + off), VP(at), 8192, None) == INVALID
        assert b"norm" in dss.lib().dss_last_error()
