"""Log probabilities, entropies and alternatives on the GPU against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from paper_2608_02560_amd import precog as P

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _check(logits, token, top, got=None):
    """Sums of V terms in fp32: lanes of up to V / 64 terms, each exponential
    good to 2^-21, so log sums within 2^-20 and a last rounding of the result;
    the entropy's terms are larger by |x - m| <= 64, with like signs."""
    T, V = logits.shape
    dev = logits if logits.is_cuda else logits.to(DEV)
    lp, ent, ids, tops = got if got is not None else P.score_tokens(
        dev, None if token is None else token.to(DEV), top=top)
    host = logits.detach().cpu()
    for t in range(T):
        r = oracle.score(host[t], None if token is None else int(token[t]), top)
        if token is not None:
            _near(lp[t].item(), r[0], 2.0 ** -20 + 2.0 ** -23 * abs(r[0]))
        _near(ent[t].item(), r[1], 2.0 ** -18 * (1 + abs(r[1])))
        if top:
            assert np.array_equal(ids[t].cpu().numpy(), r[2]), t
            for a, b in zip(tops[t].cpu().tolist(), r[3]):
                _near(a, b, 2.0 ** -20 + 2.0 ** -23 * abs(b))


def _near(a, b, tol):
    if not np.isfinite(b):
        assert a == b or (np.isnan(a) and np.isnan(b)), (a, b)
    else:
        assert abs(a - b) <= tol, (a, b, tol)


def _logits(T, V, dtype, seed, std=2.5):
    return (torch.randn((T, V), generator=torch.Generator().manual_seed(seed)) * std).to(dtype)


@pytest.mark.parametrize("V", [1, 2, 7, 8, 63, 64, 511, 512, 513, 2047, 2049, 5001, 33333])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("top", [0, 5])
def test_vocabularies(V, dtype, top):
    T = 5
    token = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(V)).int()
    _check(_logits(T, V, dtype, V), token, top)


@pytest.mark.parametrize("T", [1, 3, 300, 2100])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_rows(T, top):
    """One workgroup a row and several of them."""
    V = 20011 if T < 100 else 3001
    token = torch.randint(0, V, (T,), generator=torch.Generator().manual_seed(T)).int()
    x, dev = _logits(T, V, torch.bfloat16, T), None
    dev = x.to(DEV)
    got = P.score_tokens(dev, token.to(DEV), top=top)
    some = torch.arange(0, T, max(1, T // 20))
    pick = [None if g is None else g[some.to(DEV)] for g in got]
    _check(x[some], token[some], top, pick)


def test_one_long_row():
    x = _logits(2, 262147, torch.bfloat16, 1)
    _check(x, torch.tensor([0, 262146], dtype=torch.int32), 64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_ties_go_to_the_lower_token(dtype):
    x = torch.zeros((4, 9000), dtype=dtype)
    x[1, ::7] = 3.0
    x[2, 5000:] = 1.0
    x[3] = torch.arange(9000) % 2
    x[3, 100] = -0.0
    _check(x, torch.tensor([0, 7, 4999, 8999], dtype=torch.int32), 20)


def test_sorted_rows():
    """Ascending logits: every logit enters the list; descending: only the first."""
    up = torch.linspace(-5, 5, 6007)
    _check(torch.stack([up, up.flip(0)]), torch.tensor([6006, 0], dtype=torch.int32), 64)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_masks(dtype):
    V = 4100
    x = _logits(8, V, dtype, 2)
    low = torch.finfo(dtype).min
    x[0] = -np.inf                       # nothing left
    x[1] = low                           # the type's lowest value: a uniform row
    x[2, 3:] = -np.inf                   # fewer than `top` left
    x[3, ::2] = -np.inf
    x[4, 1::2] = low
    x[5, :] = -np.inf
    x[5, V - 1] = low
    x[6, 17] = float("nan")
    x[7, 17] = np.inf
    _check(x, torch.tensor([1, 1, 1, 1, 0, V - 1, 1, 17], dtype=torch.int32), 10)


def test_tokens_outside_the_vocabulary():
    x = _logits(4, 1000, torch.float32, 3)
    _check(x, torch.tensor([-1, -100, 1000, 2 ** 31 - 1], dtype=torch.int32), 3)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_strided_rows(dtype):
    wide = _logits(7, 3000, dtype, 4)
    token = torch.arange(7, dtype=torch.int32)
    _check(wide.to(DEV)[:, :2777], token, 5)
    _check(wide.to(DEV)[::3, :1003], token[:3], 5)
    odd = wide[:, :2777].contiguous()  # rows and base at any multiple of the element
    _check(odd.to(DEV)[1:], token[:6], 5)
    _check(odd.to(DEV).view(-1)[3:3 + 7 * 2000].view(7, 2000), token, 5)


@pytest.mark.parametrize("std", [1e-3, 30.0, 1e4])
def test_sharp_and_flat_rows(std):
    x = _logits(4, 8000, torch.float32, 5, std)
    _check(x, x.argmax(1).int(), 4)


def test_without_tokens():
    x = _logits(3, 500, torch.bfloat16, 6)
    lp, ent, ids, tops = P.score_tokens(x.to(DEV), top=2)
    assert lp is None
    _check(x, None, 2, (lp, ent, ids, tops))


def test_no_rows():
    lp, ent, ids, tops = P.score_tokens(torch.empty((0, 100), device=DEV),
                                        torch.empty(0, dtype=torch.int32, device=DEV), top=3)
    assert lp.shape == (0,) and ids.shape == (0, 3)
