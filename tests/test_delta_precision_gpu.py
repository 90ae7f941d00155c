"""How far the gated delta rule on the GPU is from 64 bits, beside a sequential
evaluation of the same inputs in 32 bits: over long sequences, whole and cut in
time, of every input and storage type.

Both round. Token after token in fp32 a state's element is rounded twice (2^-24 at
most, 2^-24.8 rms), 2^-21.8 over 32 tokens. The kernel's block of 32 tokens rounds
the operands of K S, Q S and K^T U to 22 bits (2^-23 at most, 2^-23.8 rms), leaves
out the product of two low halves of fp32 inputs (2^-22 at most) and does the rest
in fp32: 2^-21.5 rms, 1.2 times as much.  A call in segments goes through that twice
more (Phi and F) and through Phi S + F: at most twice as much.  Some more for terms
that are larger than their sum, which the two forms sum differently: four times."""
import numpy as np
import pytest
import torch

from layer_testutil import HALF, delta_inputs, delta_oracle, on_gpu, starts_of
from paper_2608_02560_amd import precog as P

pytestmark = pytest.mark.gpu
DEV = "cuda"
TIMES = 4


def _in_fp32(d, lens, h0, norm, eps=np.float32(1e-6)):
    q, k, v, g, beta = (d[n].float().numpy() for n in ("q", "k", "v", "g", "beta"))
    (T, Hk, K), (Hv, V) = k.shape, v.shape[1:]
    head = np.arange(Hv) // (Hv // Hk)
    if norm:
        q, k = (x / np.sqrt((x * x).sum(-1, keepdims=True) + eps) for x in (q, k))
    q, k, scale = q[:, head], k[:, head], np.float32(K ** -0.5)
    o, last, at = np.zeros((T, Hv, V), np.float32), [], 0
    for b, n in enumerate(lens):
        S = np.zeros((Hv, K, V), np.float32) if h0 is None else h0[b].float().numpy().copy()
        for t in range(at, at + n):
            S *= np.exp(g[t])[:, None, None]
            u = beta[t][:, None] * (v[t] - np.matmul(k[t][:, None], S)[:, 0])
            S += k[t][:, :, None] * u[:, None]
            o[t] = scale * np.matmul(q[t][:, None], S)[:, 0]
        last.append(S)
        at += n
    assert o.dtype == np.float32 and S.dtype == np.float32
    return o, np.stack(last)


def _rms(x):
    return np.sqrt(np.mean(np.square(x))) if x.size else 0.0


def _as_near(got, plain, ref, what):
    """got's error beyond half a step of its type is at most TIMES the 32-bit form's,
    in its rms (fp32) and in its largest."""
    g = got.detach().cpu().double().numpy()
    err, base = np.abs(g - ref), np.abs(plain.astype(np.float64) - ref)
    if got.dtype == torch.float32:
        assert _rms(err) <= TIMES * _rms(base), (what, _rms(err) / _rms(base))
    else:
        err = np.maximum(err - HALF[got.dtype] * (1 + 2.0 ** -7) * np.abs(ref) - 2.0 ** -25, 0)
    assert err.max() <= TIMES * base.max(), (what, err.max() / base.max())


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("lens,Hk,Hv,K,V,out,st,segments", [
    ([2500], 1, 1, 64, 48, torch.float32, torch.float32, True),
    ([2111], 1, 2, 128, 40, torch.float32, torch.float32, True),
    ([2080], 1, 1, 128, 200, torch.bfloat16, torch.float16, True),
    ([0, 13000, 1, 31, 33, 0], 1, 2, 40, 72, torch.float32, torch.float32, True),
    ([6000, 5999], 1, 2, 96, 64, torch.bfloat16, torch.float32, True),
    ([1500, 700], 4, 36, 64, 32, torch.float32, torch.float32, False),
    ([1100], 22, 66, 128, 16, torch.bfloat16, torch.float32, False)])
def test_long_sequences(lens, Hk, Hv, K, V, out, st, segments, dtype, norm):
    assert (P.delta_workspace_bytes(P.delta_desc(len(lens), sum(lens), Hk, Hv, K, V), True) > 0) == segments
    d = delta_inputs(sum(lens), Hk, Hv, K, V, 201, dtype, unit=not norm)
    h0 = (torch.randn((len(lens), Hv, K, V), generator=torch.Generator().manual_seed(202)) * 0.5).to(st)
    c = on_gpu(d)
    o, hT = P.delta(c["q"], c["k"], c["v"], c["g"], c["beta"], h0.to(DEV), starts=starts_of(lens).to(DEV), qk_norm=norm,
                    out_dtype=out, state_dtype=st)
    ro, rS = delta_oracle(d, lens, h0, qk_norm=norm)
    po, pS = _in_fp32(d, lens, h0, norm)
    _as_near(o, po, ro, "o")
    live = [b for b, n in enumerate(lens) if n]
    _as_near(hT[live], pS[live], rS[live], "hT")
