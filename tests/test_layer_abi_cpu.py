"""What the gated-delta layer's entry points refuse, on the host alone."""
import ctypes

import pytest
import torch

from paper_2608_02560_amd import precog as P

OK, ENULL, ESHAPE, EDTYPE, ESTRIDE, EALIGN, EWS = 0, 1, 2, 3, 4, 5, 6
FAKE = 0x10000


def _ref(d):
    return None if d is None else ctypes.byref(d)


def _delta(desc, q=FAKE, k=FAKE, v=FAKE, g=FAKE, beta=FAKE, starts=None, h0=None, rows=0, idx=None, o=FAKE,
           hT=FAKE + 0x100000, ws=None, nbytes=0):
    return P.lib().precog_delta_encode(_ref(desc), q, k, v, g, beta, starts, h0, rows, idx, o, hT, ws, nbytes, None)


def _step(desc, q=FAKE, k=FAKE, v=FAKE, g=FAKE, beta=FAKE, states=FAKE, rows=4, slots=FAKE, o=FAKE):
    return P.lib().precog_delta_step(_ref(desc), q, k, v, g, beta, states, rows, slots, o, None)


def _conv(desc, x=FAKE, w=FAKE, bias=None, starts=None, tail0=None, rows=0, idx=None, y=FAKE, tailT=None):
    return P.lib().precog_conv_encode(_ref(desc), x, w, bias, starts, tail0, rows, idx, y, tailT, None)


def _conv_step(desc, x=FAKE, w=FAKE, bias=None, tails=FAKE, rows=4, slots=FAKE, y=FAKE):
    return P.lib().precog_conv_step(_ref(desc), x, w, bias, tails, rows, slots, y, None)


def _score(T=4, V=1000, stride=0, dtype=P.BF16, logits=FAKE, token=FAKE, top=2, lp=FAKE, ent=FAKE, ids=FAKE,
           tlp=FAKE, ws=FAKE, nbytes=1 << 20):
    return P.lib().precog_score_tokens(logits, dtype, T, V, stride, token, top, lp, ent, ids, tlp, ws, nbytes, None)


@pytest.mark.parametrize("bad,code", [
    (dict(batch=-1), ESHAPE), (dict(seqlen=-1), ESHAPE), (dict(batch=1 << 31), ESHAPE), (dict(seqlen=1 << 31), ESHAPE),
    (dict(batch=1 << 20, seqlen=1 << 20), ESHAPE), (dict(batch=1 << 28, seqlen=1), ESHAPE),
    (dict(k_heads=0), ESHAPE), (dict(v_heads=0), ESHAPE), (dict(v_heads=3), ESHAPE), (dict(k_heads=1 << 17), ESHAPE),
    (dict(k_dim=0), ESHAPE), (dict(k_dim=136), ESHAPE), (dict(k_dim=12), ESHAPE), (dict(v_dim=264), ESHAPE),
    (dict(v_dim=4), ESHAPE), (dict(in_dtype=P.F16), EDTYPE), (dict(out_dtype=P.F16), EDTYPE),
    (dict(state_dtype=P.BF16), EDTYPE), (dict(in_dtype=7), EDTYPE),
    (dict(q_stride=120), ESTRIDE), (dict(k_stride=-8), ESTRIDE), (dict(v_stride=248), ESTRIDE),
    (dict(q_stride=132), EALIGN), (dict(v_stride=1 << 25), ESTRIDE), (dict(h0_batch_stride=64 * 64), ESTRIDE),
    (dict(hT_batch_stride=4 * 64 * 64 + 4), EALIGN), (dict(eps=-1.0), ESHAPE), (dict(eps=float("nan")), ESHAPE),
    (dict(scale=float("inf")), ESHAPE)])
def test_delta_descriptors(bad, code):
    good = dict(batch=2, seqlen=16, k_heads=2, v_heads=4, k_dim=64, v_dim=64)
    assert _delta(P.delta_desc(**{**good, **bad})) == code
    if not set(bad) & {"batch", "seqlen", "hT_batch_stride"} or bad.get("batch") == -1:
        assert _step(P.delta_desc(**{**good, **bad})) == code


def test_delta_arguments():
    good = P.delta_desc(2, 16, 2, 4, 64, 64)
    assert _delta(None) == ENULL
    for name in ("q", "k", "v"):
        assert _delta(good, **{name: None}) == ENULL
    for name in ("q", "k", "v", "h0", "o", "hT"):
        assert _delta(good, **{name: FAKE + 8}) == EALIGN
    for name in ("g", "beta"):
        assert _delta(good, **{name: FAKE + 2}) == EALIGN
    assert _delta(good, starts=FAKE + 2) == EALIGN
    assert _delta(good, h0=FAKE, rows=3, idx=FAKE + 1) == EALIGN
    assert _delta(good, idx=FAKE, rows=-1) == ESHAPE
    assert _delta(good, idx=FAKE, rows=3) == ENULL               # rows need a store
    # states only partly in place
    row = 4 * 64 * 64 * 4
    assert _delta(good, h0=FAKE, hT=FAKE + row) == ESTRIDE
    assert _delta(good, h0=FAKE, rows=2, idx=FAKE, hT=FAKE) == ESTRIDE
    assert _delta(good, h0=FAKE, hT=FAKE + 16) == ESTRIDE
    layers = P.delta_desc(2, 16, 2, 4, 64, 64, h0_batch_stride=3 * 4 * 64 * 64, hT_batch_stride=3 * 4 * 64 * 64)
    assert _delta(layers, h0=FAKE, hT=FAKE + row // 2) == ESTRIDE


def test_delta_workspace():
    long = P.delta_desc(1, 40000, 2, 4, 128, 128)
    need = P.delta_workspace_bytes(long)
    assert need > 0 and need == P.delta_workspace_bytes(long, True)
    assert _delta(long) == EWS and _delta(long, ws=FAKE, nbytes=need - 1) == EWS
    assert _delta(long, ws=FAKE + 8, nbytes=need) == EALIGN
    for d in (P.delta_desc(2, 16, 2, 4, 64, 64), P.delta_desc(0, 40000, 2, 4, 64, 64),
              P.delta_desc(64, 40000, 2, 4, 64, 64), P.delta_desc(1, 40000, 2, 3, 64, 64),
              P.delta_desc(1, 40000, 33, 66, 64, 64), P.delta_desc(1, 2000, 2, 4, 64, 64),
              P.delta_desc(1 << 20, 1 << 20, 1, 1, 64, 64)):
        assert P.delta_workspace_bytes(d) == 0


def test_nothing_to_do_is_ok_without_a_gpu():
    assert _delta(P.delta_desc(0, 16, 2, 4, 64, 64), q=None, k=None, v=None) == OK
    assert _delta(P.delta_desc(2, 16, 2, 4, 64, 64), o=None, hT=None) == OK
    assert _delta(P.delta_desc(2, 0, 2, 4, 64, 64), q=None, k=None, v=None, hT=None) == OK
    assert _step(P.delta_desc(0, 1, 2, 4, 64, 64), q=None) == OK
    assert _step(P.delta_desc(3, 1, 2, 4, 64, 64), states=None, rows=0) == OK
    assert _conv(P.conv_desc(0, 5, 64, 4), x=None) == OK
    assert _conv(P.conv_desc(2, 5, 0, 4), x=None) == OK
    assert _conv(P.conv_desc(2, 5, 64, 4), y=None) == OK
    assert _conv_step(P.conv_desc(3, 1, 64, 4), tails=None, rows=0) == OK
    assert _score(T=0, logits=None) == OK
    assert _score(token=None, ent=None, top=0) == OK


def test_step_arguments():
    good = P.delta_desc(3, 1, 2, 4, 64, 64)
    assert _step(None) == ENULL
    for name in ("q", "k", "v", "states", "slots"):
        assert _step(good, **{name: None}) == ENULL
    for name in ("q", "k", "v", "states", "o"):
        assert _step(good, **{name: FAKE + 8}) == EALIGN
    for name in ("g", "beta", "slots"):
        assert _step(good, **{name: FAKE + 2}) == EALIGN
    assert _step(good, rows=-1) == ESHAPE
    assert _step(P.delta_desc(65536, 1, 2, 4, 64, 64)) == ESHAPE
    assert _step(P.delta_desc(65535, 1, 1, 8192, 8, 8)) == ESHAPE


@pytest.mark.parametrize("bad,code", [
    (dict(batch=-1), ESHAPE), (dict(dim=-8), ESHAPE), (dict(seqlen=-1), ESHAPE), (dict(width=1), ESHAPE),
    (dict(width=5), ESHAPE), (dict(dim=60), EALIGN), (dict(x_stride=56), ESTRIDE), (dict(x_stride=68), EALIGN),
    (dict(in_dtype=P.F16), EDTYPE), (dict(out_dtype=P.F16), EDTYPE), (dict(batch=1 << 20, seqlen=1 << 20), ESHAPE)])
def test_conv_descriptors(bad, code):
    good = dict(batch=2, seqlen=16, dim=64, width=4)
    assert _conv(P.conv_desc(**{**good, **bad})) == code
    if not set(bad) & {"seqlen"}:
        assert _conv_step(P.conv_desc(**{**good, **bad})) == code


def test_conv_arguments():
    good = P.conv_desc(2, 16, 64, 4)
    assert _conv(None) == ENULL and _conv_step(None) == ENULL
    assert _conv(good, x=None) == ENULL and _conv(good, w=None) == ENULL
    assert _conv(good, tail0=None, rows=3, idx=FAKE) == ENULL
    assert _conv(good, tail0=FAKE, rows=-3, idx=FAKE) == ESHAPE
    for name in ("x", "w", "bias", "tail0", "y", "tailT"):
        assert _conv(good, **{name: FAKE + 8}) == EALIGN
    assert _conv(good, starts=FAKE + 1) == EALIGN
    assert _conv(good, tail0=FAKE, tailT=FAKE + 16) == ESTRIDE
    assert _conv(good, tail0=FAKE, rows=4, idx=FAKE, tailT=FAKE) == ESTRIDE
    for name in ("x", "w", "tails", "slots"):
        assert _conv_step(good, **{name: None}) == ENULL
    assert _conv_step(good, slots=FAKE + 2) == EALIGN
    assert _conv_step(good, rows=-1) == ESHAPE


def test_score_arguments():
    assert _score(T=-1) == ESHAPE and _score(V=0) == ESHAPE and _score(top=65) == ESHAPE and _score(top=-1) == ESHAPE
    assert _score(T=1 << 31) == ESHAPE and _score(V=(1 << 28) + 1) == ESHAPE
    assert _score(dtype=5) == EDTYPE
    assert _score(stride=999) == ESTRIDE
    for name in ("logits", "lp", "ids", "tlp"):
        assert _score(**{name: None}) == ENULL
    for name, off in (("logits", 1), ("token", 2), ("lp", 2), ("ent", 2), ("ids", 2), ("tlp", 2), ("ws", 8)):
        assert _score(**{name: FAKE + off}) == EALIGN
    need = P.score_workspace_bytes(1, 100000, 5)
    assert need > 0
    assert _score(T=1, V=100000, top=5, ws=None) == EWS
    assert _score(T=1, V=100000, top=5, nbytes=need - 1) == EWS
    assert P.score_workspace_bytes(-1, 5, 5) == 0 and P.score_workspace_bytes(0, 5, 5) == 0
    assert P.score_workspace_bytes(100000, 50000, 64) == 0


def test_wrappers_refuse_host_tensors():
    x = torch.zeros((2, 3, 1, 64))
    with pytest.raises(ValueError):
        P.delta(x, x, x)
    with pytest.raises(ValueError):
        P.delta_step(x[0], x[0], x[0], None, None, torch.zeros((4, 1, 64, 64)), torch.zeros(3, dtype=torch.int32))
    with pytest.raises(ValueError):
        P.conv(x[:, :, 0], torch.zeros((64, 4)))
    with pytest.raises(ValueError):
        P.score_tokens(torch.zeros((2, 100)))


def test_token_strides():
    base = torch.zeros((6, 4, 100))
    assert P._token_stride("t", base[:, :, :64], 2) == 100
    assert P._token_stride("t", base, 2) == 0
    assert P._token_stride("t", base[0, :, 8:72].unflatten(1, (2, 32)), 1) == 100
    assert P._token_stride("t", base[:, ::2], 2) == 200
    assert P._token_stride("t", base[:, :1, :64], 2) == 400   # one token a row
    assert P._token_stride("t", base[:1, :, :64], 2) == 100
    assert P._token_stride("t", base[0, :1, :64], 1) == 0
    for t, lead in ((torch.zeros(1, 64).expand(5, 64), 1), (torch.zeros(1, 4, 64).expand(3, 4, 64), 2),
                    (torch.zeros(5, 1, 64).expand(5, 2, 64), 1)):
        with pytest.raises(ValueError):
            P._token_stride("t", t, lead)           # the same elements for several tokens
    with pytest.raises(ValueError):
        P._token_stride("t", base.transpose(1, 2), 2)
    with pytest.raises(ValueError):
        P._token_stride("t", base[:, :3], 2)  # rows of the batch do not follow one another
