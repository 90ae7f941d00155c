"""Calls of the gated-delta layer and of token scoring with more threads than one
launch can hold are refused on the host."""
import pytest

from paper_2608_02560_amd import precog as P
from test_layer_abi_cpu import ESHAPE, EWS, FAKE, OK, _conv, _delta, _score, _step


def _past(status):
    """Past the checks of arguments: what the device check says where there is no GPU."""
    return status not in (OK, ESHAPE, EWS)


gpu_free = pytest.mark.skipif("__import__('torch').cuda.is_available()", reason="must not launch on made-up pointers")


@gpu_free
@pytest.mark.parametrize("dtype,K,V,most", [
    (P.BF16, 64, 128, (2 ** 32 - 1) // (8 * 64)), (P.BF16, 128, 32, (2 ** 32 - 1) // (5 * 64)),
    (P.F32, 128, 96, (2 ** 32 - 1) // (4 * 64)), (P.F32, 64, 8, (2 ** 32 - 1) // (4 * 64)),
    (P.BF16, 64, 256, (2 ** 32 - 1) // (8 * 64) // 2), (P.BF16, 64, 160, (2 ** 32 - 1) // (8 * 64) // 2)])
def test_delta(dtype, K, V, most):
    """4 chain waves of 32 columns at most, and 4, 3 or 1 that prepare."""
    assert _past(_delta(P.delta_desc(most, 1, 1, 1, K, V, dtype)))
    assert _delta(P.delta_desc(most + 1, 1, 1, 1, K, V, dtype)) == ESHAPE
    assert _delta(P.delta_desc(most + 1, 1, 1, 1, K, V, dtype), o=None, hT=None) == OK
    assert _delta(P.delta_desc(1 << 20, 1, 16, 64, K, V, dtype)) == ESHAPE


@gpu_free
def test_step():
    assert _past(_step(P.delta_desc(65535, 1, 1, 256, 8, 8)))
    assert _step(P.delta_desc(65535, 1, 1, 257, 8, 8)) == ESHAPE
    assert _step(P.delta_desc(65535, 1, 1, 129, 8, 136)) == ESHAPE


@gpu_free
def test_conv():
    n = (2 ** 32 - 1) // 64
    assert _conv(P.conv_desc(1, 2 ** 31 - 1, 8, 4), starts=FAKE) == ESHAPE   # 2^26 runs of 64 threads: 2^32
    assert _past(_conv(P.conv_desc(1, 2 ** 31 - 32, 8, 4), starts=FAKE))      # a run less
    assert _conv(P.conv_desc(5, 2 ** 31 - 32, 8, 4), starts=FAKE, tailT=FAKE) == ESHAPE
    assert _past(_conv(P.conv_desc(n, 0, 8, 4), starts=FAKE, tailT=FAKE))
    assert _conv(P.conv_desc(n + 1, 0, 8, 4), starts=FAKE, tailT=FAKE) == ESHAPE
    assert _past(_conv(P.conv_desc(n - 1, 32, 8, 4), starts=FAKE, tailT=FAKE))
    assert _conv(P.conv_desc(n, 32, 8, 4), starts=FAKE, tailT=FAKE) == ESHAPE
    assert _past(_conv(P.conv_desc(n, 32, 8, 4), starts=FAKE, tail0=FAKE, tailT=FAKE))     # in place: two launches
    assert _conv(P.conv_desc(1, 2 ** 30, 2048, 4), starts=FAKE) == ESHAPE
    assert _past(_conv(P.conv_desc(1, 2 ** 29 - 32, 2048, 4), starts=FAKE))


@gpu_free
def test_score():
    assert _past(_score(T=2 ** 24 - 1, V=2)) and _score(T=2 ** 24, V=2) == ESHAPE
    assert _score(T=2 ** 24, V=2, token=None, ent=None, top=0) == OK
