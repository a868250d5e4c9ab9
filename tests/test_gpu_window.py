"""focus_window_attn_fwd and focus_window_attn_bwd against the definition in 64 bits (bounds: window_ref.py)."""
import math

import pytest
import torch

from paper_2604_03260_amd import focus
from tests.window_ref import TORCH, check, reference

pytestmark = pytest.mark.gpu


def rows(B, H, n, d, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(B, H, n, d, generator=g, device="cuda") * scale).to(TORCH[dtype])


def run(p, q, k, v, dout=None, spans=None, fill=float("nan")):
    out = torch.full_like(q, fill)
    lse = torch.full(q.shape[:3], fill, device="cuda")
    focus.focus_window_attn_fwd(p, q, k, v, out, lse, spans=spans)
    if dout is None:
        return out, lse
    ws = focus.alloc_window_bwd_workspace(p)
    ws.fill_(255)                                      # (NaN wherever it is read before it is written)
    grads = [torch.full_like(x, fill) for x in (q, k, v)]
    focus.focus_window_attn_bwd(p, q, k, v, out, lse, dout, ws, *grads, spans=spans)
    return (out, lse) + tuple(grads)


NAMES = ("out", "lse", "dq", "dk", "dv")

# B, Hq, Hkv, n, d, window, sinks, softcap: one row, odd lengths, windows of one row and past the end, sinks behind
# the window, in it, as many as the sequence; grouped heads 1, 2, 3, 4, 5, 8
CASES = [
    (1, 4, 4, 1, 64, 1, 0, 0.0), (2, 4, 1, 2, 128, 1, 1, 0.0), (1, 8, 2, 33, 64, 7, 2, 0.0), (2, 3, 1, 64, 80, 64, 0, 0.0),
    (1, 10, 2, 127, 96, 20, 5, 20.0), (1, 2, 2, 128, 128, 1000, 3, 0.0), (1, 16, 2, 129, 128, 32, 129, 0.0),
    (1, 4, 1, 300, 256, 65, 40, 0.0), (2, 6, 3, 517, 64, 100, 1, 5.0), (1, 4, 1, 1000, 128, 257, 70, 0.0),
    (1, 1, 1, 2100, 64, 128, 200, 0.0), (1, 5, 1, 700, 80, 1, 3, 0.0), (1, 4, 2, 1537, 96, 511, 130, 30.0),
    (3, 12, 12, 257, 64, 128, 4, 0.0), (1, 2, 1, 400, 256, 400, 10, 10.0), (1, 8, 1, 3001, 128, 300, 4, 0.0),
]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CASES)
def test_forward_and_gradients(case, dtype):
    B, Hq, Hkv, n, d, w, s, cap = case
    q, k, v, g = (rows(B, h, n, d, dtype, i) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    p = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype, softcap=cap)
    got = run(p, q, k, v, g)
    for b in range(B):
        ref = reference(q[b], k[b], v[b], w, s, 1 / math.sqrt(d), cap, dtype, g[b])
        for name, x in zip(NAMES, got):
            check(x[b], ref, name)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_large_logits_and_a_rising_reference(dtype):
    """Logits up to some hundreds whose largest come late in the walk, and a scale of its own."""
    B, Hq, Hkv, n, d, w, s = 1, 4, 2, 400, 64, 150, 3
    q, k, v, g = (rows(B, h, n, d, dtype, 10 + i) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    k = (k * torch.linspace(0.1, 6, n, device="cuda")[:, None]).to(k.dtype)
    p = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype, scale=0.5)
    got = run(p, q, k, v, g)
    ref = reference(q[0], k[0], v[0], w, s, 0.5, 0.0, dtype, g[0])
    for name, x in zip(NAMES, got):
        check(x[0], ref, name)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("packed", [False, True])
def test_spans(packed, dtype):
    """Sequences of all lengths, one of them empty, some out of the tensors' range: rows in no span stay as they were, and what
    they hold (NaN here) reaches nothing."""
    Hq, Hkv, d, w, s = 4, 2, 64, 50, 3
    if packed:
        n, want = 900, [(10, 1), (20, 0), (40, 333), (400, 64), (500, 129), (890, 10)]
        given = want[:5] + [(890, 999), (-5, 3), (900, 4), (70, -1)]
        want = want + [(0, 0)] * 3
    else:
        n, want = 300, [(0, 300), (100, 200), (0, 1), (299, 1), (7, 0), (50, 129)]
        given = want
    B = len(given)
    Bt = 1 if packed else B
    q, k, v, g = (rows(Bt, h, n, d, dtype, 20 + i) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    used = torch.zeros(Bt, n, dtype=torch.bool, device="cuda")
    for b, (first, length) in enumerate(want):
        used[0 if packed else b, first:first + length] = True
    for x in (q, k, v, g):
        x[~used[:, None].expand(x.shape[:3])] = float("nan")
    spans = torch.tensor(given, dtype=torch.int32, device="cuda")
    p = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype, packed=packed, span_max=0 if not packed else 500)
    got = run(p, q, k, v, g, spans, fill=7.0)
    for name, x in zip(NAMES, got):
        rest = x[~used[:, None].expand(x.shape[:3])]
        assert (rest == 7.0).all(), name
    for b, (first, length) in enumerate(want):
        t, r = 0 if packed else b, slice(first, first + length)
        if length:
            ref = reference(q[t, :, r], k[t, :, r], v[t, :, r], w, s, 1 / 8.0, 0.0, dtype, g[t, :, r])
            for name, x in zip(NAMES, got):
                check(x[t, :, r], ref, name)


def test_spans_are_cut_to_the_longest_promised():
    q, k, v, g = (rows(1, 2, 400, 64, "bf16", 30 + i) for i in range(4))
    spans = torch.tensor([[0, 400]], dtype=torch.int32, device="cuda")
    p = focus.make_window_params(1, 2, 2, 400, 64, 30, sinks=2, span_max=150)
    got = run(p, q, k, v, g, spans, fill=7.0)
    for x in got:
        assert (x[:, :, 150:] == 7.0).all()
    ref = reference(q[0, :, :150], k[0, :, :150], v[0, :, :150], 30, 2, 1 / 8.0, 0.0, "bf16", g[0, :, :150])
    for name, x in zip(NAMES, got):
        check(x[0, :, :150], ref, name)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 80), ("f32", 96), ("bf16", 256)])
def test_strided_tensors(dtype, d):
    """q, k, v and their gradients as views of a packed projection, out and dout as [B,n,H,d]: the bytes of the contiguous run."""
    B, Hq, Hkv, n, w, s = 2, 6, 2, 203, 40, 3
    x = rows(B, n, Hq + 2 * Hkv, d, dtype, 40).permute(0, 2, 1, 3)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    g = rows(B, n, Hq, d, dtype, 41).permute(0, 2, 1, 3)
    grads = torch.full((B, n, Hq + 2 * Hkv, d), 7.0, dtype=x.dtype, device="cuda").permute(0, 2, 1, 3)
    out, lse = torch.empty(B, n, Hq, d, dtype=x.dtype, device="cuda").permute(0, 2, 1, 3), torch.empty(B, Hq, n, device="cuda")
    p = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype, q_strides=focus.strides_of(q), kv_strides=focus.strides_of(k),
                                 o_strides=focus.strides_of(out))
    focus.focus_window_attn_fwd(p, q, k, v, out, lse)
    focus.focus_window_attn_bwd(p, q, k, v, out, lse, g, focus.alloc_window_bwd_workspace(p), grads[:, :Hq], grads[:, Hq:Hq + Hkv],
                                grads[:, Hq + Hkv:])
    p2 = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype)
    want = run(p2, q.contiguous(), k.contiguous(), v.contiguous(), g.contiguous())
    for a, b in zip((out, lse, grads[:, :Hq], grads[:, Hq:Hq + Hkv], grads[:, Hq + Hkv:]), want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_values_that_are_not_finite_stay_with_those_that_see_them(value, dtype):
    """Row 70 of k and v (then of q and dout) is not finite: rows that do not see it (keys it does not see) give the bytes of a clean run."""
    B, Hq, Hkv, n, d, w, s = 1, 2, 1, 260, 64, 40, 3
    q, k, v, g = (rows(B, h, n, d, dtype, 50 + i) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    p = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype)
    clean = run(p, q, k, v, g)
    i = torch.arange(n, device="cuda")
    for where in ("k", "v"):
        k2, v2 = k.clone(), v.clone()
        (k2 if where == "k" else v2)[0, 0, 70, 5] = value
        got = run(p, q, k2, v2, g)
        apart = (i < 70) | (i >= 70 + w)               # rows that do not see key 70
        for j in (0, 1, 2):
            assert torch.equal(got[j][:, :, apart], clean[j][:, :, apart]), (where, NAMES[j])
        lost = ~torch.isfinite(got[0].float()).all(-1)
        shows = (~apart).expand(lost.shape)
        if where == "k" and math.isinf(value):         # (a logit of -inf is a weight of zero: such a row is finite by the definition)
            shows = shows & (q[..., 5] > 0)
        assert lost[shows].all(), "a row that sees it shows it"
        # keys that no spoiled row sees
        far = (i < 70 - w + 1) & (i >= s) | (i >= 70 + w)
        for j in (3, 4):
            assert torch.equal(got[j][:, :, far], clean[j][:, :, far]), (where, NAMES[j])
    out, lse = clean[:2]
    for where in ("q", "dout"):
        q2, g2 = q.clone(), g.clone()
        (q2 if where == "q" else g2)[0, 0, 70, 5] = value
        grads = [torch.empty_like(x) for x in (q, k, v)]
        focus.focus_window_attn_bwd(p, q2, k, v, out, lse, g2, focus.alloc_window_bwd_workspace(p), *grads)
        apart = (i > 70) | (i <= 70 - w)
        apart[:s] = False
        assert torch.equal(grads[0][:, :, i != 70], clean[2][:, :, i != 70])
        for j in (1, 2):
            assert torch.equal(grads[j][:, :, apart], clean[2 + j][:, :, apart]), (where, j)
            if not (where == "q" and math.isinf(value)):      # (an infinite query may give probabilities of zero)
                assert not torch.isfinite(grads[1][:, :, 70 - w + 1:71].float()).all(-1).any()


def test_gradients_against_differences():
    """The directional derivatives of sum(out * g) in 32 bits.  f is a sum of some hundreds of terms, each off by about 2^-22; over a step of 2h =
    0.02 that is 1e-3, and h^2 times the third derivative is below 1e-3 too."""
    B, Hq, Hkv, n, d, w, s, cap = 1, 4, 2, 90, 64, 20, 3, 8.0
    q, k, v, g = (rows(B, h, n, d, "f32", 60 + i) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    p = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype="f32", softcap=cap)
    grads = run(p, q, k, v, g)[2:]
    f = lambda *a: (run(p, *a)[0].double() * g.double()).sum().item()
    for i in range(3):
        e = rows(B, (Hq, Hkv, Hkv)[i], n, d, "f32", 70 + i)
        e /= e.norm()
        plus, minus = [q, k, v], [q, k, v]
        plus[i], minus[i] = plus[i] + 0.01 * e, minus[i] - 0.01 * e
        got = (f(*plus) - f(*minus)) / 0.02
        assert abs(got - (grads[i].double() * e.double()).sum().item()) <= 5e-3


def test_a_long_sequence_against_rows_of_the_definition():
    """40000 rows, far chunks of the sinks in several work-groups: sampled rows, and the gradients of the sinks and of sampled keys."""
    Hq, Hkv, n, d, w, s = 4, 1, 40000, 128, 700, 70
    q, k, v, g = (rows(1, h, n, d, "bf16", 80 + i) for i, h in enumerate((Hq, Hkv, Hkv, Hq)))
    p = focus.make_window_params(1, Hq, Hkv, n, d, w, sinks=s)
    out, lse, dq, dk, dv = run(p, q, k, v, g)
    scale, u = 1 / math.sqrt(d), 2.0 ** -8
    qd, kd, vd, gd = (x[0].double() for x in (q, k, v, g))
    gdk, gdv, adk, adv = (torch.zeros(n, d, dtype=torch.float64, device="cuda") for _ in range(4))
    for i0 in range(0, n, 1000):
        a0 = max(0, i0 - w + 1)
        cols = torch.cat([torch.arange(min(s, a0), device="cuda"), torch.arange(a0, i0 + 1000, device="cuda")])
        r = torch.arange(i0, i0 + 1000, device="cuda")[:, None]
        see = (cols <= r) & ((r - cols < w) | (cols < s))
        for h in range(Hq):
            x = (qd[h, i0:i0 + 1000] @ kd[0, cols].T * scale).masked_fill(~see, -math.inf)
            l = torch.logsumexp(x, -1)
            pr = torch.exp(x - l[:, None])
            o = pr @ vd[0, cols]
            assert ((out[0, h, i0:i0 + 1000].double() - o).abs() <= u * o.abs() + 1.1 * u * (pr @ vd[0, cols].abs()) + 1e-4).all()
            assert ((lse[0, h, i0:i0 + 1000].double() - l).abs() <= 1e-4).all()
            gr = gd[h, i0:i0 + 1000]
            ds = pr * (gr @ vd[0, cols].T - (gr * o).sum(-1, keepdim=True)) * scale
            # out is rounded (and its products are), which moves delta: the bound of dS, see window_ref.py
            eds = 1.1 * u * ds.abs() + 1.1 * pr * scale * (gr.abs() * (u * o.abs() + 1.1 * u * (pr @ vd[0, cols].abs()))).sum(-1, keepdim=True)
            want = ds @ kd[0, cols]
            assert ((dq[0, h, i0:i0 + 1000].double() - want).abs() <= u * want.abs() + eds @ kd[0, cols].abs() + 1e-4).all()
            gdk.index_add_(0, cols, ds.T @ qd[h, i0:i0 + 1000])
            adk.index_add_(0, cols, eds.T @ qd[h, i0:i0 + 1000].abs())
            gdv.index_add_(0, cols, pr.T @ gr)
            adv.index_add_(0, cols, 1.1 * u * (pr.T @ gr.abs()))
    assert ((dk[0, 0].double() - gdk).abs() <= u * gdk.abs() + adk + 1e-3).all()
    assert ((dv[0, 0].double() - gdv).abs() <= u * gdv.abs() + adv + 1e-3).all()


def test_same_bits_every_time_and_on_other_streams():
    q, k, v, g = (rows(1, h, 1500, 128, "bf16", 90 + i) for i, h in enumerate((8, 2, 2, 8)))
    p = focus.make_window_params(1, 8, 2, 1500, 128, 200, sinks=5)
    first = run(p, q, k, v, g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        second = run(p, q, k, v, g)
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)


def test_replay_from_a_graph_with_new_inputs():
    Hq, Hkv, n, d = 4, 2, 700, 96
    make = lambda seed: [rows(1, h, n, d, "f16", seed + i) for i, h in enumerate((Hq, Hkv, Hkv, Hq))]
    args = make(100)
    p = focus.make_window_params(1, Hq, Hkv, n, d, 90, sinks=3, dtype="f16")
    ws = focus.alloc_window_bwd_workspace(p)
    outs = [torch.empty_like(args[0]), torch.empty(1, Hq, n, device="cuda")] + [torch.empty_like(x) for x in args[:3]]

    def step():
        focus.focus_window_attn_fwd(p, *args[:3], outs[0], outs[1])
        focus.focus_window_attn_bwd(p, *args[:3], outs[0], outs[1], args[3], ws, *outs[2:])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for rep in range(3):
        for x, y in zip(args, make(110 + 10 * rep)):
            x.copy_(y)
        for x in outs:
            x.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(outs, run(p, *args)):
            assert torch.equal(x, y)


# Calls with so many rows that a work-group has four pieces of 32 rows (the others share one piece; the choice goes by the number of
# work-groups): the cases above are small.  Groups of 3 heads leave wavefronts of a work-group at different rows.
@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("d", [64, 80, 96, 128, 256])
@pytest.mark.parametrize("cap", [0.0, 15.0])
def test_forward_of_many_rows(d, dtype, cap):
    B, Hq, Hkv, n, w, s = 8, 9, 3, 517, 65, 40
    q, k, v = (rows(B, h, n, d, dtype, 80 + i) for i, h in enumerate((Hq, Hkv, Hkv)))
    p = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype, softcap=cap)
    got = run(p, q, k, v)
    for b in range(B):
        ref = reference(q[b], k[b], v[b], w, s, 1 / math.sqrt(d), cap, dtype)
        for name, x in zip(NAMES, got):
            check(x[b], ref, name)


@pytest.mark.parametrize("dtype,d", [("bf16", 64), ("f16", 128), ("f32", 64)])
def test_spans_of_many_rows(dtype, d):
    Hq, Hkv, w, s = 12, 4, 50, 3
    lengths = [1, 333, 0, 64, 129, 2, 31, 600, 33, 128, 0, 7] * 3
    gap, want, at = 3, [], 0
    for x in lengths:
        want.append((at, x))
        at += x + gap
    q, k, v = (rows(1, h, at, d, dtype, 90 + i) for i, h in enumerate((Hq, Hkv, Hkv)))
    used = torch.zeros(at, dtype=torch.bool, device="cuda")
    for first, length in want:
        used[first:first + length] = True
    for x in (q, k, v):
        x[:, :, ~used] = float("nan")
    p = focus.make_window_params(len(want), Hq, Hkv, at, d, w, sinks=s, dtype=dtype, packed=True, span_max=600)
    got = run(p, q, k, v, spans=torch.tensor(want, dtype=torch.int32, device="cuda"), fill=7.0)
    for name, x in zip(NAMES, got):
        assert (x[:, :, ~used] == 7.0).all(), name
    for first, length in want:
        if length:
            r = slice(first, first + length)
            ref = reference(q[0, :, r], k[0, :, r], v[0, :, r], w, s, 1 / math.sqrt(d), 0.0, dtype)
            for name, x in zip(NAMES, got):
                check(x[0, :, r], ref, name)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
def test_values_that_are_not_finite_among_many_rows(value, dtype):
    B, Hq, Hkv, n, d, w, s = 48, 6, 3, 260, 64, 40, 3
    q, k, v = (rows(B, h, n, d, dtype, 100 + i) for i, h in enumerate((Hq, Hkv, Hkv)))
    p = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype)
    clean = run(p, q, k, v)
    i = torch.arange(n, device="cuda")
    apart = (i < 70) | (i >= 70 + w)
    for where in ("k", "v"):
        k2, v2 = k.clone(), v.clone()
        (k2 if where == "k" else v2)[5, 1, 70, 5] = value
        got = run(p, q, k2, v2)
        sees = torch.zeros(B, Hq, n, dtype=torch.bool, device="cuda")
        sees[5, 2:4] = ~apart
        for j in (0, 1):
            assert torch.equal(got[j][~sees], clean[j][~sees]), (where, NAMES[j])
        if where == "k" and math.isinf(value):
            sees &= q[..., 5] > 0
        assert (~torch.isfinite(got[0].float()).all(-1))[sees].all()


def test_short_calls_replayed_from_a_graph():
    """A call of few rows in a graph, with new inputs and eager calls between the replays."""
    B, H, n, d, w = 1, 8, 200, 64, 33
    q, k, v = (rows(B, H, n, d, "bf16", 110 + i) for i in range(3))
    p = focus.make_window_params(B, H, H, n, d, w, sinks=2)
    out, lse = run(p, q, k, v)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(stream):
        with torch.cuda.graph(graph, stream=stream):
            focus.focus_window_attn_fwd(p, q, k, v, out, lse)
    torch.cuda.synchronize()
    for i in range(4):
        for j, x in enumerate((q, k, v)):
            x.copy_(rows(B, H, n, d, "bf16", 120 + 3 * i + j))
        graph.replay()
        want = run(p, q, k, v)
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
