"""The gated-delta layer's operators as they are used together: a retrieved
chunk's state and tail injected into the query's convolution and delta rule,
the answer's tokens scored, and the session continued token by token; the same
steps captured in a HIP graph, on other streams and beside one another."""
import numpy as np
import pytest
import torch

import oracle
from layer_testutil import O16, check, delta_bar, starts_of
from paper_2608_02560_amd import precog as P

pytestmark = pytest.mark.gpu
DEV = "cuda"

HK, HV, K, V, W = 2, 4, 64, 64, 4
NK, NV = HK * K, HV * V
D = 2 * NK + NV
VOCAB = 1003


def _weights(seed):
    g = torch.Generator().manual_seed(seed)
    return dict(conv=torch.randn((D, W), generator=g) * W ** -0.5,
                out=torch.randn((NV, VOCAB), generator=g) * NV ** -0.5 * 4)


def _tokens(n, seed):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((n, D), generator=g)
    gate = -0.3 * torch.nn.functional.softplus(torch.randn((n, HV), generator=g))
    beta = torch.sigmoid(torch.randn((n, HV), generator=g))
    token = torch.randint(0, VOCAB, (n,), generator=g).int()
    return dict(x=x, g=gate, beta=beta, token=token)


def _split(y):
    return (y[:, :NK].unflatten(1, (HK, K)), y[:, NK:2 * NK].unflatten(1, (HK, K)), y[:, 2 * NK:].unflatten(1, (HV, V)))


def _layer(w, t, starts, tails, states, idx):
    y, tail = P.conv(t["x"], w["conv"], None, tails, starts=starts, tail_idx=idx)
    q, k, v = _split(y)
    o, hT = P.delta(q, k, v, t["g"], t["beta"], states, starts=starts, h0_idx=idx, qk_norm=True)
    logits = o.reshape(-1, NV) @ w["out"]
    return tail, hT, o, P.score_tokens(logits, t["token"], top=5)


def _step(w, t, tails, states, slots, o=None):
    y = P.conv_step(t["x"], w["conv"], None, tails, slots)
    q, k, v = _split(y)
    o = P.delta_step(q, k, v, t["g"], t["beta"], states, slots, qk_norm=True)
    return o, P.score_tokens(o.reshape(-1, NV) @ w["out"], t["token"], top=5)


def _oracle_layer(w, t, tail, state):
    y, tail = oracle.conv(t["x"], w["conv"], None, tail)
    q, k, v = y[:, :NK].reshape(-1, HK, K), y[:, NK:2 * NK].reshape(-1, HK, K), y[:, 2 * NK:].reshape(-1, HV, V)
    o, state = oracle.delta(q, k, v, t["g"], t["beta"], state, qk_norm=True)
    logits = o.reshape(-1, NV) @ w["out"].double().numpy()
    return tail, state, o, [oracle.score(x, int(n), 5) for x, n in zip(logits, t["token"])]


def _dev(d):
    return {n: t.to(DEV) for n, t in d.items()}


def _check_scores(got, ref):
    """Logits here are sums of NV products of an o good to delta_bar and of size
    up to 16: off by up to 5 sqrt(2) delta_bar of that beside their own fp32 sums."""
    lp, ent, ids, tops = (t.cpu() for t in got)
    tol = 2e-3
    for i, (a, e, best, _) in enumerate(ref):
        assert abs(lp[i] - a) < tol and abs(ent[i] - e) < tol
        # a logit within tol of another may change places with it
        same = ids[i].numpy() == best
        assert same.all() or np.abs(np.diff(ref[i][3])).min() < tol


def test_query_from_a_retrieved_chunk_and_its_continuation():
    w = _weights(1)
    wd = _dev(w)
    # three chunks are encoded into tails and states, keyed by embeddings
    lens = [70, 33, 129]
    chunks = _tokens(sum(lens), 2)
    tail, hT, _, _ = _layer(wd, _dev(chunks), starts_of(lens).to(DEV), None, None, None)
    keys = torch.nn.functional.normalize(torch.randn((3, 64), generator=torch.Generator().manual_seed(3)), dim=1)
    query = torch.nn.functional.normalize(keys[[2, 0]] + 0.02, dim=1)
    idx = P.top1(query.to(DEV), keys.to(DEV))
    assert idx.tolist() == [2, 0]
    # two queries run from what they retrieved
    qlens = [9, 40]
    queries = _tokens(sum(qlens), 4)
    qtail, qstate, o, scores = _layer(wd, _dev(queries), starts_of(qlens).to(DEV), tail, hT, idx)

    def part(t, a, b):
        return {n: x[a:b] for n, x in t.items()}

    at = np.concatenate([[0], np.cumsum(lens)])
    qat = np.concatenate([[0], np.cumsum(qlens)])
    refs, ro, rs = [], [], []
    for i, c in enumerate((2, 0)):
        rt, rst, _, _ = _oracle_layer(w, part(chunks, at[c], at[c + 1]), None, None)
        rt, rst, oo, sc = _oracle_layer(w, part(queries, qat[i], qat[i + 1]), rt, rst)
        refs.append((rt, rst))
        ro.append(oo)
        rs += sc
    bar = 3 * delta_bar(200)  # y's own rounding (2^-19) enters q, k and v
    check(o, np.concatenate(ro), bar, "o")
    check(qstate, np.stack([r[1] for r in refs]), bar, "states")
    assert torch.allclose(qtail.cpu().double(), torch.tensor(np.stack([r[0] for r in refs])))
    _check_scores(scores, rs)

    # and go on as sessions, in a table of slots
    tails = torch.zeros((6, W - 1, D), device=DEV)
    states = torch.zeros((6, HV, K, V), device=DEV)
    slots = torch.tensor([4, 1], dtype=torch.int32, device=DEV)
    tails[slots.long()], states[slots.long()] = qtail, qstate
    for s in range(5):
        t = _tokens(2, 10 + s)
        o, sc = _step(wd, _dev(t), tails, states, slots)
        for i in range(2):
            rt, rst, oo, rsc = _oracle_layer(w, part(t, i, i + 1), *refs[i])
            refs[i] = (rt, rst)
            check(o[i], oo[0], bar, "step")
            _check_scores([x[i:i + 1] for x in sc], rsc)


def test_decode_step_graph_replays_equal_eager():
    """A padded decode batch captured once and replayed with other sessions in
    its slots, eager work between the replays."""
    n, rows = 8, 12
    w = _dev(_weights(20))
    g = torch.Generator().manual_seed(21)
    tails = torch.randn((rows, W - 1, D), generator=g).to(DEV)
    states = torch.randn((rows, HV, K, V), generator=g).to(DEV)
    static = _dev(_tokens(n, 22))
    slots = torch.zeros(n, dtype=torch.int32, device=DEV)

    def fresh(seed):
        r = np.random.default_rng(seed)
        s = r.permutation(rows)[:n].astype(np.int32)
        s[r.integers(0, n)] = -1  # padding
        return _dev(_tokens(n, seed)), torch.tensor(s, device=DEV)

    t, s = fresh(23)
    slots.copy_(s)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(w, static, tails.clone(), states.clone(), slots)  # warm-up
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go, gs = _step(w, static, tails, states, slots)
    for rep in range(5):
        t, s = fresh(30 + rep)
        for name in static:
            static[name].copy_(t[name])
        slots.copy_(s)
        et, es = tails.clone(), states.clone()
        eo, esc = _step(w, t, et, es, s)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        live = (s >= 0).cpu()
        assert torch.equal(tails, et) and torch.equal(states, es)
        assert torch.equal(go[live], eo[live])
        for a, b in zip(gs, esc):
            assert torch.equal(a[live], b[live])


def test_prefill_graph_replays_equal_eager():
    """Sequence lengths are data on the device: a captured prefill serves other
    lengths and other retrieved rows."""
    w = _dev(_weights(40))
    T, B, rows = 90, 3, 5
    g = torch.Generator().manual_seed(41)
    tails = torch.randn((rows, W - 1, D), generator=g).to(DEV)
    states = torch.randn((rows, HV, K, V), generator=g).to(DEV)
    static = _dev(_tokens(T, 42))
    starts = starts_of([30, 30, 30]).to(DEV)
    idx = torch.zeros(B, dtype=torch.int32, device=DEV)
    _layer(w, static, starts, tails, states, idx)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = _layer(w, static, starts, tails, states, idx)
    for rep, lens in enumerate(([30, 30, 30], [1, 60, 29], [0, 90, 0], [64, 0, 20])):
        t = _dev(_tokens(T, 50 + rep))
        for name in static:
            static[name].copy_(t[name])
        starts.copy_(starts_of(lens).to(DEV))
        idx.copy_(torch.tensor([rep, 4 - rep, 2], dtype=torch.int32))
        eager = _layer(w, t, starts, tails, states, idx)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        n = sum(lens)
        assert torch.equal(out[0], eager[0]) and torch.equal(out[1], eager[1])
        assert torch.equal(out[2][:n], eager[2][:n])
        for a, b in zip(out[3], eager[3]):
            assert torch.equal(a[:n], b[:n])


def test_segmented_prefill_graph_replays_equal_eager():
    """A long sequence in time segments, captured with its workspace; two graphs
    of it side by side."""
    lens = [2300, 1900]
    sets = [_dev(_tokens(sum(lens), 90 + i)) for i in range(3)]
    starts = starts_of(lens).to(DEV)
    static = [{n: t.clone() for n, t in sets[0].items()} for _ in range(2)]

    def run(t):
        q, k, v = _split(t["x"])
        return P.delta(q, k, v, t["g"], t["beta"], starts=starts, qk_norm=True, out_dtype=torch.bfloat16)

    run(static[0])
    graphs, outs = [], []
    for s in static:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(s))
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in range(2)]
    for rep in range(4):
        pick = [sets[(rep + i) % 3] for i in range(2)]
        for s, t in zip(static, pick):
            for n in s:
                s[n].copy_(t[n])
        eager = [run(t) for t in pick]
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, eager):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


@pytest.mark.parametrize("as_int", [False, True])
def test_other_streams(as_int):
    """Two streams at once, named by argument, while the current one is neither."""
    w = _dev(_weights(60))
    g = torch.Generator(device=DEV).manual_seed(61)
    logits = [torch.randn((3, 70001), generator=g, device=DEV) for _ in range(2)]
    sets = [_dev(_tokens(200, 62 + i)) for i in range(2)]
    starts = starts_of([120, 80]).to(DEV)

    def run(t, x, stream=None):
        y, _ = P.conv(t["x"], w["conv"], starts=starts, stream=stream)
        q, k, v = _split(y)
        o, hT = P.delta(q, k, v, t["g"], t["beta"], starts=starts, qk_norm=True, stream=stream)
        return [o, hT] + list(P.score_tokens(x, t["token"][:3], top=3, stream=stream))

    ref = [run(t, x) for t, x in zip(sets, logits)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(3):
        got = [run(t, x, s.cuda_stream if as_int else s) for t, x, s in zip(sets, logits, streams)]
    torch.cuda.synchronize()
    for a, b in zip(got, ref):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


def test_offsets_past_32_bits():
    """Rows of a state store, of a tail store, of logits and of packed tokens
    whose element offsets do not fit 32 bits."""
    big = (1 << 31) // (HV * K * V) + 8
    store = torch.empty((big, HV, K, V), dtype=torch.float16, device=DEV)
    row = torch.randn((HV, K, V), device=DEV).half()
    store[big - 2] = row
    t = _dev(_tokens(40, 70))
    q, k, v = (x.contiguous() for x in _split(t["x"]))
    idx = torch.tensor([big - 2], dtype=torch.int32, device=DEV)
    starts = starts_of([40]).to(DEV)
    a = P.delta(q, k, v, t["g"], t["beta"], store, starts=starts, h0_idx=idx, qk_norm=True)
    b = P.delta(q, k, v, t["g"], t["beta"], row[None], starts=starts, qk_norm=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    small = row[None].clone()
    one = {n: x[:1] for n, x in dict(q=q, k=k, v=v, g=t["g"], beta=t["beta"]).items()}
    oa = P.delta_step(one["q"], one["k"], one["v"], one["g"], one["beta"], store, idx, qk_norm=True)
    ob = P.delta_step(one["q"], one["k"], one["v"], one["g"], one["beta"], small,
                      torch.zeros(1, dtype=torch.int32, device=DEV), qk_norm=True)
    assert torch.equal(oa, ob) and torch.equal(store[big - 2], small[0])
    del store

    dim = 8192
    big = (1 << 31) // (3 * dim) + 8
    tails = torch.empty((big, 3, dim), dtype=torch.bfloat16, device=DEV)
    tails[big - 3] = torch.randn((3, dim), device=DEV).bfloat16()
    x = torch.randn((5, dim), device=DEV).bfloat16()
    cw = torch.randn((dim, 4), device=DEV)
    idx = torch.tensor([big - 3], dtype=torch.int32, device=DEV)
    a = P.conv(x, cw, None, tails, starts=starts_of([5]).to(DEV), tail_idx=idx)
    b = P.conv(x, cw, None, tails[big - 3:big - 2].clone(), starts=starts_of([5]).to(DEV))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    del tails

    T, n = 18000, 120001
    logits = torch.empty((T, n), dtype=torch.bfloat16, device=DEV)
    logits.zero_()
    logits[T - 2:] = torch.randn((2, n), device=DEV).bfloat16()
    tok = torch.full((T,), 7, dtype=torch.int32, device=DEV)
    a = P.score_tokens(logits, tok, top=3)
    b = P.score_tokens(logits[T - 2:].clone(), tok[:2], top=3)
    assert torch.equal(a[2][T - 2:], b[2])
    assert torch.allclose(a[0][T - 2:], b[0], rtol=0, atol=1e-5) and torch.allclose(a[1][T - 2:], b[1], rtol=0, atol=1e-5)
    del logits

    T = (1 << 31) // D + 200
    x = torch.empty((T, D), dtype=torch.bfloat16, device=DEV)
    x[T - 70:] = torch.randn((70, D), device=DEV).bfloat16()
    gates = torch.zeros((T, HV), device=DEV)
    starts = torch.tensor([T - 70, T - 30, T], dtype=torch.int32, device=DEV)
    q, k, v = _split(x)
    a = P.delta(q, k, v, gates, None, starts=starts, qk_norm=True, out_dtype=torch.bfloat16)
    q, k, v = _split(x[T - 70:].clone())
    b = P.delta(q, k, v, gates[:70], None, starts=starts_of([40, 30]).to(DEV), qk_norm=True, out_dtype=torch.bfloat16)
    # the many tokens have the first call computed in segments: equal but for rounding
    check(a[0][T - 70:], b[0].double().cpu().numpy(), O16)
    check(a[1], b[1].double().cpu().numpy(), 2 * delta_bar(40))
    cw = torch.randn((D, 4), device=DEV)
    a = P.conv(x, cw, starts=starts)
    b = P.conv(x[T - 70:].clone(), cw, starts=starts_of([40, 30]).to(DEV))
    assert torch.equal(a[0][T - 70:], b[0]) and torch.equal(a[1], b[1])


def test_refusals_of_the_wrappers():
    t = _dev(_tokens(6, 80))
    q, k, v = _split(t["x"])
    g, beta = t["g"], t["beta"]
    s = starts_of([6]).to(DEV)
    h0 = torch.zeros((1, HV, K, V), device=DEV)

    def bad(fn):
        with pytest.raises((ValueError, P.PrecogError)):
            fn()

    bad(lambda: P.delta(q.half(), k.half(), v.half(), g, beta, starts=s))
    bad(lambda: P.delta(q, k.bfloat16(), v, g, beta, starts=s))
    bad(lambda: P.delta(q, k, v, g.half(), beta, starts=s))
    bad(lambda: P.delta(q, k, v, g, beta[:, :2], starts=s))
    bad(lambda: P.delta(q, k, v[:5], g, beta, starts=s))
    bad(lambda: P.delta(q, k, v, g, beta, starts=s.long()))
    bad(lambda: P.delta(q, k, v, g, beta, starts=s.cpu()))
    bad(lambda: P.delta(q, k, v, g, beta, h0.double(), starts=s))
    bad(lambda: P.delta(q, k, v, g, beta, h0[:, :2], starts=s))
    bad(lambda: P.delta(q, k, v, g, beta, h0.transpose(2, 3), starts=s, state_dtype=torch.bfloat16))
    bad(lambda: P.delta(q, k, v, g, beta, starts=s, h0_idx=s[:1]))
    bad(lambda: P.delta(q, k, v, g, beta, starts=s, out_dtype=torch.float16))
    bad(lambda: P.delta(None, k, v, g, beta, starts=s))
    bad(lambda: P.delta(q[:, :, :60], k[:, :, :60], v, g, beta, starts=s))
    bad(lambda: P.delta(q[..., 1:57], k[..., 1:57], v, g, beta, starts=s))
    bad(lambda: P.delta_step(q, k, v, g, beta, h0, s))
    bad(lambda: P.delta_step(q, k, v, g, beta, h0.cpu(), torch.zeros(6, dtype=torch.int32, device=DEV)))
    bad(lambda: P.conv(t["x"][:, :60], torch.zeros((60, 4), device=DEV), starts=s))
    bad(lambda: P.conv(t["x"], torch.zeros((D, 5), device=DEV), starts=s))
    bad(lambda: P.conv(t["x"], torch.zeros((D, 4), device=DEV), torch.zeros(D - 1, device=DEV), starts=s))
    bad(lambda: P.conv_step(t["x"], torch.zeros((D, 4), device=DEV), None, torch.zeros((2, 4, D), device=DEV),
                            torch.zeros(6, dtype=torch.int32, device=DEV)))
    bad(lambda: P.score_tokens(t["x"], t["token"].long()))
    bad(lambda: P.score_tokens(t["x"], t["token"][:3]))
    bad(lambda: P.score_tokens(t["x"], t["token"], top=65))
    bad(lambda: P.score_tokens(t["x"], t["token"], top=-1))
    bad(lambda: P.score_tokens(t["x"].t(), None, top=1))
    bad(lambda: P.score_tokens(t["x"][:1].expand(6, D), t["token"]))
