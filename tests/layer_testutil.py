"""Inputs, oracle runs and tolerances of the gated-delta layer's tests."""
from __future__ import annotations

import math

import numpy as np
import torch

import oracle

# Half a step of a storage type, relative to the value.
HALF = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def delta_bar(tokens):
    """Relative error that 32-bit arithmetic may leave in o and in the states
    after `tokens` tokens (before the rounding to their storage type), against
    the rms of the result.

    A block of 32 tokens passes six products whose operands carry 22 bits (or
    32 tokens' fp32 sums of up to 128 terms, sqrt(32 * 128) 2^-25 = 2^-19: the
    same order): independent errors of at most 2^-21 each, 2^-21 sqrt(6 / 3) =
    2^-20.5 rms.  The rule never expands (|I - beta k k^T| <= 1 for |k| <= 1 and
    0 <= beta <= 1, a <= 1), so blocks add at most in squares: times
    sqrt(1 + tokens / 32).  The largest of up to 10^6 errors lies within five
    of their rms."""
    return 5 * 2.0 ** -20.5 * math.sqrt(1 + tokens / 32)


# What a bf16 o may have more than delta_bar, against its rms: its two terms Q S
# and Q K^T U take operands of 11 bits, rounded by at most 2^-11 (half a step of
# 2^-10), 2^-11 / sqrt(3) rms: S in the one, two of them in the other, together
# 2^-11 of the terms' rms, which are up to 1.5 times o's where they partly cancel;
# five times that is 2^-8.1.
O16 = 2.0 ** -8


def check(got, ref, bar, what=""):
    """|got - ref| <= half a step of got's type + bar * max(|ref|, rms(ref))."""
    t = got.dtype
    g = got.detach().cpu().double().numpy()
    r = np.asarray(ref, dtype=np.float64)
    assert g.shape == r.shape, (what, g.shape, r.shape)
    if r.size == 0:
        return
    fine = np.isfinite(r)
    assert np.array_equal(np.isnan(g), np.isnan(r)), what
    inf = ~fine & ~np.isnan(r)
    assert np.array_equal(g[inf], r[inf]), what
    g, r = g[fine], r[fine]
    if r.size == 0:
        return
    rms = float(np.sqrt(np.mean(r * r)))
    tiny = {torch.float16: 2.0 ** -25}.get(t, 0.0)  # half a step of subnormals
    tol = HALF[t] * (1 + 2.0 ** -7) * np.abs(r) + tiny + bar * np.maximum(np.abs(r), rms)
    worst = np.max(np.abs(g - r) / np.maximum(tol, 1e-300))
    assert worst <= 1.0, "%s: %.2f times the tolerance" % (what, worst)


def delta_inputs(tokens, Hk, Hv, K, V, seed, dtype=torch.bfloat16, unit=False, sliced=True,
                 rate=(0.002, 0.7)):
    """q, k, v (slices of one tensor), g, beta on the CPU."""
    gen = torch.Generator().manual_seed(seed)
    nk, nv = Hk * K, Hv * V
    mixed = torch.randn((tokens, 2 * nk + nv), generator=gen)
    if unit:
        qk = mixed[:, :2 * nk].reshape(tokens, 2 * Hk, K)
        mixed[:, :2 * nk] = (qk / qk.norm(dim=-1, keepdim=True).clamp_min(1e-9)).reshape(tokens, 2 * nk)
    mixed = mixed.to(dtype)
    q, k, v = mixed[:, :nk], mixed[:, nk:2 * nk], mixed[:, 2 * nk:]
    if not sliced:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    r = torch.exp(torch.linspace(math.log(rate[0]), math.log(rate[1]), Hv))
    g = -r * torch.nn.functional.softplus(torch.randn((tokens, Hv), generator=gen))
    beta = torch.sigmoid(torch.randn((tokens, Hv), generator=gen) * 2)
    return dict(q=q.unflatten(1, (Hk, K)), k=k.unflatten(1, (Hk, K)), v=v.unflatten(1, (Hv, V)), g=g,
                beta=beta)


def on_gpu(d):
    """Copies to the GPU that keep slices slices (of a copy of their base)."""
    out, bases = {}, {}
    for n, t in d.items():
        if t is None:
            out[n] = None
            continue
        s = t.untyped_storage()
        if s.data_ptr() not in bases:
            whole = torch.empty(0, dtype=t.dtype).set_(s)
            bases[s.data_ptr()] = whole.cuda()
        out[n] = bases[s.data_ptr()].as_strided(t.shape, t.stride(), t.storage_offset())
    return out


def delta_oracle(d, lens, h0=None, **kw):
    """(o of all tokens, states [B, ...]) of packed sequences."""
    o, S, at = [], [], 0
    for b, n in enumerate(lens):
        part = {name: None if t is None else t[at:at + n] for name, t in d.items()}
        oo, ss = oracle.delta(part["q"], part["k"], part["v"], part["g"], part["beta"],
                              None if h0 is None else h0[b], **kw)
        o.append(oo)
        S.append(ss)
        at += n
    return (None if d["q"] is None else np.concatenate(o)), np.stack(S)


def starts_of(lens, first=0):
    return torch.tensor(np.concatenate([[first], first + np.cumsum(lens)]), dtype=torch.int32)
