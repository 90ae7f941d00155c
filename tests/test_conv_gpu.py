"""The short causal convolution on the GPU against the fp64 oracle."""
import numpy as np
import pytest
import torch

import oracle
from layer_testutil import check, starts_of
from paper_2608_02560_amd import precog as P

pytestmark = pytest.mark.gpu
DEV = "cuda"

# W products and W sums of fp32 (2 W 2^-24 of the terms' size, up to a few
# times the rms), an exponential good to 2^-21 for |y| below 16 and a division
BAR = 2.0 ** -19


def _inputs(tokens, D, W, dtype, seed, bias=True):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn((tokens, D), generator=g).to(dtype), torch.randn((D, W), generator=g) * W ** -0.5,
            torch.randn((D,), generator=g) if bias else None)


def _tails(rows, W, D, dtype, seed):
    return torch.randn((rows, W - 1, D), generator=torch.Generator().manual_seed(seed)).to(dtype)


def _dev(t):
    return None if t is None else t.to(DEV)


def _oracle(x, w, bias, lens, tails, silu=True):
    y, tl, at = [], [], 0
    for b, n in enumerate(lens):
        a, c = oracle.conv(x[at:at + n], w, bias, None if tails is None else tails[b], silu)
        y.append(a)
        tl.append(c)
        at += n
    return np.concatenate(y), np.stack(tl)


@pytest.mark.parametrize("lens", [[1], [2], [3, 1, 2], [32], [33], [0, 5, 0, 0, 70, 0], [31, 97, 128, 1], [700]])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_lengths(lens, W, dtype):
    D = 72
    x, w, bias = _inputs(sum(lens), D, W, dtype, 1)
    tails = _tails(len(lens), W, D, dtype, 2)
    y, t = P.conv(_dev(x), _dev(w), _dev(bias), _dev(tails), starts=starts_of(lens).to(DEV))
    ry, rt = _oracle(x, w, bias, lens, tails)
    check(y, ry, BAR)
    assert torch.equal(t.cpu().double(), torch.tensor(rt))


@pytest.mark.parametrize("D", [8, 512, 520, 2048, 3000])
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("silu", [True, False])
def test_channels(D, out, silu):
    lens = [40, 3]
    x, w, bias = _inputs(sum(lens), D, 4, torch.bfloat16, 3, bias=silu)
    y, t = P.conv(_dev(x), _dev(w), _dev(bias), starts=starts_of(lens).to(DEV), silu=silu, out_dtype=out)
    ry, rt = _oracle(x, w, bias, lens, None, silu)
    check(y, ry, BAR)
    assert torch.equal(t.cpu().double(), torch.tensor(rt))


def test_padded_batch_and_strided_inputs():
    B, L, D, W = 3, 50, 64, 4
    x, w, bias = _inputs(B * L, 2 * D, W, torch.bfloat16, 4)
    w, bias = w[:D].contiguous(), bias[:D].contiguous()
    part = _dev(x)[:, D:].unflatten(0, (B, L))  # a slice of a wider projection
    y, t = P.conv(part, _dev(w), _dev(bias))
    ry, rt = _oracle(x[:, D:], w, bias, [L] * B, None)
    check(y.view(B * L, D), ry, BAR)
    assert torch.equal(t.cpu().double(), torch.tensor(rt))


def test_stored_tails():
    lens, D, W = [4, 0, 1, 60], 128, 4
    x, w, _ = _inputs(sum(lens), D, W, torch.bfloat16, 5)
    store = _tails(6, W, D, torch.bfloat16, 6)
    idx = torch.tensor([5, 2, -1, 5], dtype=torch.int32)
    y, t = P.conv(_dev(x), _dev(w), None, _dev(store), starts=starts_of(lens).to(DEV), tail_idx=_dev(idx))
    ry, rt = _oracle(x, w, None, lens, store[idx.clamp(min=0).long()])
    check(y[:4], ry[:4], BAR)
    assert torch.isnan(y[4]).all()  # its tail is in no row
    check(y[5:], ry[5:], BAR)
    for b in (0, 1, 3):
        assert torch.equal(t[b].cpu().double(), torch.tensor(rt[b]))
    assert torch.isnan(t[2, :2]).all() and torch.equal(t[2, 2].cpu(), x[4])


@pytest.mark.parametrize("lens", [[200, 2, 0, 64], [1, 1]])
def test_tails_in_place(lens):
    D, W = 256, 4
    x, w, bias = _inputs(sum(lens), D, W, torch.bfloat16, 7)
    tails = _tails(len(lens), W, D, torch.bfloat16, 8)
    dev = _dev(tails)
    y, t = P.conv(_dev(x), _dev(w), _dev(bias), dev, starts=starts_of(lens).to(DEV), tailT=dev)
    assert t is dev
    ry, rt = _oracle(x, w, bias, lens, tails)
    check(y, ry, BAR)
    assert torch.equal(t.cpu().double(), torch.tensor(rt))


def test_rows_outside_the_sequences_stay():
    T, D = 100, 64
    x, w, _ = _inputs(T, D, 3, torch.float32, 9)
    starts = torch.tensor([7, 40, 40, 90], dtype=torch.int32, device=DEV)
    y = torch.full((T, D), 9.0, device=DEV)
    P.conv_encode(P.conv_desc(3, T, D, 3, P.F32, P.F32), _dev(x), _dev(w), None, starts, y=y)
    ry, _ = _oracle(x[7:90], w, None, [33, 0, 50], None)
    assert (y[:7] == 9).all() and (y[90:] == 9).all()
    check(y[7:90], ry, BAR)


def test_only_tails():
    lens, D = [5, 2], 64
    x, w, _ = _inputs(sum(lens), D, 4, torch.bfloat16, 10)
    y, t = P.conv(_dev(x), _dev(w), None, starts=starts_of(lens).to(DEV), want_y=False)
    assert y is None
    assert torch.equal(t.cpu().double(), torch.tensor(_oracle(x, w, None, lens, None)[1]))


def test_large_inputs_saturate_as_the_function_does():
    x = torch.tensor([[-300.0, -90.0, 90.0, 300.0, 0.0, -20.0, 20.0, 1e30]], device=DEV).repeat(3, 1)
    w = torch.zeros((8, 2), device=DEV)
    w[:, 1] = 1.0
    y, _ = P.conv(x, w, None, starts=starts_of([3]).to(DEV))
    ref = torch.tensor([[0.0, -90.0 * np.exp(-90.0), 90.0, 300.0, 0.0, -20.0 / (1 + np.exp(20.0)), 20.0, 1e30]])
    assert torch.allclose(y[1:].cpu().double(), ref.repeat(2, 1), rtol=1e-5, atol=1e-30)


# ---------------------------------------------------------------- single tokens
@pytest.mark.parametrize("n,D", [(1, 8), (7, 520), (100, 4096)])
@pytest.mark.parametrize("W", [2, 3, 4])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_step(n, D, W, dtype):
    x, w, bias = _inputs(n, D, W, dtype, 20)
    tails = _tails(n + 2, W, D, dtype, 21)
    slots = np.random.default_rng(3).permutation(n + 2)[:n].astype(np.int32)
    dev = _dev(tails)
    y = P.conv_step(_dev(x), _dev(w), _dev(bias), dev, torch.tensor(slots, device=DEV), out_dtype=torch.float32)
    rt = tails.double().numpy().copy()
    ry = np.empty((n, D))
    for i, s in enumerate(slots):
        ry[i:i + 1], rt[s] = oracle.conv(x[i:i + 1], w, bias, rt[s])
    check(y, ry, BAR)
    assert torch.equal(dev.cpu().double(), torch.tensor(rt))


def test_step_odd_slots():
    n, D, W = 7, 64, 4
    x, w, _ = _inputs(n, D, W, torch.bfloat16, 22)
    tails = _tails(4, W, D, torch.bfloat16, 23)
    slots = np.array([3, -1, 1, 3, 4, 3, 1], dtype=np.int32)
    dev, y = _dev(tails), torch.full((n, D), 5.0, device=DEV)
    P.conv_step_raw(P.conv_desc(n, 1, D, W, P.BF16, P.F32), _dev(x), _dev(w), None, dev, 4,
                    torch.tensor(slots, device=DEV), y)
    rt, ry = tails.double().numpy().copy(), np.full((n, D), 5.0)
    for i, s in enumerate(slots):
        if 0 <= s < 4:
            ry[i:i + 1], rt[s] = oracle.conv(x[i:i + 1], w, None, rt[s])
    check(y, ry, BAR)
    assert torch.equal(dev.cpu().double(), torch.tensor(rt))
