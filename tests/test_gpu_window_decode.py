"""focus_window_cache_fill and focus_window_decode_step_at against the definition in 64 bits (bounds: window_ref.py), and the operators in
a row as a layer uses them."""
import math

import pytest
import torch

from paper_2604_03260_amd import focus
from tests.test_gpu_window import rows, run
from tests.window_ref import TORCH, check, reference

pytestmark = pytest.mark.gpu


def row_of(pos, cap, s):
    return pos if pos < cap else s + (pos - s) % (cap - s)


# B, Hq, Hkv, d, window, sinks, capacity, softcap
CASES = [(1, 8, 2, 64, 1, 0, 1, 0.0), (2, 4, 4, 128, 20, 3, 23, 0.0), (3, 5, 1, 80, 33, 0, 40, 10.0), (1, 64, 1, 128, 300, 7, 333, 0.0),
         (2, 6, 2, 96, 64, 130, 194, 0.0), (1, 4, 2, 256, 100, 1, 128, 0.0), (4, 12, 12, 64, 1000, 4, 600, 0.0), (1, 80, 2, 64, 31, 2, 64, 0.0)]


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
@pytest.mark.parametrize("case", CASES)
def test_steps_follow_the_definition(case, dtype):
    """A whole sequence in memory; the caches hold what was written at each position, NaN where nothing was; each sequence of the batch
    stands elsewhere, one is skipped."""
    B, Hq, Hkv, d, w, s, cap, softcap = case
    rolls = cap - s >= w
    total = 3 * cap + 10 if rolls else cap
    q, k, v = (rows(B, h, total, d, dtype, i) for i, h in enumerate((Hq, Hkv, Hkv)))
    p = focus.make_window_params(B, Hq, Hkv, cap, d, w, sinks=s, dtype=dtype, softcap=softcap)
    ws = focus.alloc_window_decode_workspace(p)
    stops = sorted({0, 1, s - 1, s, s + 1, w, cap - 2, cap - 1, cap, cap + 1, total // 2, total - 1} & set(range(total)))
    for t in stops:
        pos = [(t + 5 * b) % total for b in range(B)]
        kc = torch.full((B, Hkv, cap, d), float("nan"), dtype=q.dtype, device="cuda")
        vc = kc.clone()
        for b in range(B):
            for x in range(max(0, pos[b] - cap + s), pos[b]):
                kc[b, :, row_of(x, cap, s)], vc[b, :, row_of(x, cap, s)] = k[b, :, x], v[b, :, x]
            for x in range(min(s, pos[b])):
                kc[b, :, x], vc[b, :, x] = k[b, :, x], v[b, :, x]
        k0, v0 = kc.clone(), vc.clone()
        out, lse = torch.full((B, Hq, d), 7.0, dtype=q.dtype, device="cuda"), torch.full((B, Hq), 7.0, device="cuda")
        idx = torch.arange(B, device="cuda")
        at = torch.tensor(pos, dtype=torch.int32, device="cuda")
        qn, kn, vn = (x[idx, :, at.long()].contiguous() for x in (q, k, v))
        if B > 2:
            at[1] = -1 if t % 2 else (2 ** 31 - 1 if not rolls else -7)
        focus.focus_window_decode_step_at(p, at, qn, kn, vn, kc, vc, ws, out, lse)
        for b in range(B):
            if B > 2 and b == 1:
                assert (out[b] == 7.0).all() and (lse[b] == 7.0).all()
            else:
                # (the definition over the visible keys in order, the last row's)
                seen = [x for x in range(pos[b] + 1) if x < s or pos[b] - x < w]
                ref = last_row(q[b, :, pos[b]], k[b][:, seen], v[b][:, seen], softcap, dtype)
                check(out[b], ref, "out")
                check(lse[b], ref, "lse")
                k0[b, :, row_of(pos[b], cap, s)], v0[b, :, row_of(pos[b], cap, s)] = kn[b], vn[b]
        assert torch.equal(kc.view(torch.uint8), k0.view(torch.uint8)) and torch.equal(vc.view(torch.uint8), v0.view(torch.uint8))


def last_row(q, k, v, softcap, dtype):
    """q [Hq,d] over keys k, v [Hkv,m,d], all visible: row m - 1 of a sequence whose other queries do not matter."""
    Hq, d = q.shape
    m = k.shape[1]
    full = torch.zeros(Hq, m, d, dtype=q.dtype, device="cuda")
    full[:, m - 1] = q
    r = reference(full, k, v, m, 0, 1 / math.sqrt(d), softcap, dtype)
    return {x: y[:, m - 1] for x, y in r.items()}


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("cap,n", [(300, 300), (300, 100), (64, 300), (64, 65), (64, 64), (64, 1000)])
def test_a_prompt_fills_the_caches(cap, n, dtype):
    B, Hkv, d, w, s = 3, 2, 80, 50, 4
    k, v = rows(B, Hkv, n, d, dtype, 1), rows(B, Hkv, n, d, dtype, 2)
    p = focus.make_window_params(B, 4, Hkv, n, d, w, sinks=s, dtype=dtype)
    spans = torch.tensor([[0, n], [n // 3, n - n // 3], [5, 0]], dtype=torch.int32, device="cuda")
    for sp in (None, spans):
        kc = torch.full((B, Hkv, cap, d), 7.0, dtype=k.dtype, device="cuda")
        vc = kc.clone()
        focus.focus_window_cache_fill(p, k, v, kc, vc, spans=sp)
        for b in range(B):
            first, length = (0, n) if sp is None else sp[b].tolist()
            want_k = torch.full((Hkv, cap, d), 7.0, dtype=k.dtype, device="cuda")
            want_v = want_k.clone()
            for x in range(length):
                want_k[:, row_of(x, cap, s)], want_v[:, row_of(x, cap, s)] = k[b, :, first + x], v[b, :, first + x]
            assert torch.equal(kc[b], want_k) and torch.equal(vc[b], want_v)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_a_layer_from_projection_to_generation(dtype):
    """Norms and rotation of a packed projection, window attention, caches that go round, then 40 tokens one by one from one captured
    graph: the rows of the whole sequence in one call, which is checked against the definition."""
    B, Hq, Hkv, n, d, w, s, steps = 2, 8, 2, 150, 64, 40, 3, 40
    cap, total, H = w + s + 5, 190, 12
    x = rows(B, total, H, d, dtype, 3)
    wq, wk = (1 + 0.1 * torch.randn(d, device="cuda", generator=torch.Generator(device="cuda").manual_seed(i)) for i in (4, 5))
    turns = focus.focus_rope_frequencies(d)[0].cuda()

    def front(xs, pos):
        """[B,m,H,d] -> q, k [B,.,m,d] normalised and rotated, v"""
        m = xs.shape[1]
        t = xs.permute(0, 2, 1, 3)
        q, k, v = t[:, :Hq], t[:, Hq:Hq + Hkv], t[:, Hq + Hkv:]
        rp = focus.make_rope_params(B, Hq, Hkv, m, d, d, dtype=dtype, q_strides=focus.strides_of(q), k_strides=focus.strides_of(k))
        qo, ko = torch.empty(B, Hq, m, d, dtype=xs.dtype, device="cuda"), torch.empty(B, Hkv, m, d, dtype=xs.dtype, device="cuda")
        focus.focus_qk_norm_rope(rp, q, k, wq, wk, pos, turns, qo, ko)
        return qo, ko, v.contiguous()
    whole = front(x, None)
    wp = focus.make_window_params(B, Hq, Hkv, total, d, w, sinks=s, dtype=dtype)
    out, lse = run(wp, *whole)
    refs = [reference(*(t[b] for t in whole), w, s, 1 / math.sqrt(d), 0.0, dtype) for b in range(B)]
    for b in range(B):
        check(out[b], refs[b], "out")
    q, k, v = front(x[:, :n].contiguous(), None)
    assert torch.equal(q, whole[0][:, :, :n])
    kc = torch.zeros(B, Hkv, cap, d, dtype=x.dtype, device="cuda")
    vc = torch.zeros_like(kc)
    focus.focus_window_cache_fill(focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype=dtype), k, v, kc, vc)
    dp = focus.make_window_params(B, Hq, Hkv, cap, d, w, sinks=s, dtype=dtype)
    ws = focus.alloc_window_decode_workspace(dp)
    token = torch.empty(B, 1, H, d, dtype=x.dtype, device="cuda")
    pos = torch.full((B, 1), n, dtype=torch.int32, device="cuda")
    o1, l1 = torch.empty(B, Hq, d, dtype=x.dtype, device="cuda"), torch.empty(B, Hq, device="cuda")

    def step():
        qn, kn, vn = front(token, pos)
        focus.focus_window_decode_step_at(dp, pos.view(-1), qn, kn, vn, kc, vc, ws, o1, l1)
        pos.add_(1)
    token.copy_(x[:, n:n + 1])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
        pos.fill_(n)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for t in range(n, total):
        token.copy_(x[:, t:t + 1])
        graph.replay()
        torch.cuda.synchronize()
        for b in range(B):
            check(o1[b], {y: z[:, t] for y, z in refs[b].items()}, "out")
            check(l1[b], {y: z[:, t] for y, z in refs[b].items()}, "lse")
    assert steps == total - n


def test_gradients_through_norm_rotation_and_attention():
    """A training step of the layer in 32 bits: the gradient of the packed projection against differences (the bounds of the two operators'
    own tests: 5e-3 at a step of 0.01)."""
    B, Hq, Hkv, n, d, w, s = 1, 4, 2, 70, 64, 20, 2
    x, g = rows(B, n, 8, d, "f32", 6), rows(B, Hq, n, d, "f32", 7)
    wq, wk = torch.full((d,), 1.1, device="cuda"), torch.full((d,), 0.9, device="cuda")
    turns = focus.focus_rope_frequencies(d)[0].cuda()
    st = focus.strides_of(x.permute(0, 2, 1, 3))
    rp = focus.make_rope_params(B, Hq, Hkv, n, d, d, dtype="f32", q_strides=st, k_strides=st)
    wp = focus.make_window_params(B, Hq, Hkv, n, d, w, sinks=s, dtype="f32", kv_strides=None)

    def forward(y):
        t = y.permute(0, 2, 1, 3)
        q, k = torch.empty(B, Hq, n, d, device="cuda"), torch.empty(B, Hkv, n, d, device="cuda")
        focus.focus_qk_norm_rope(rp, t[:, :Hq], t[:, Hq:Hq + Hkv], wq, wk, None, turns, q, k)
        v = t[:, Hq + Hkv:].contiguous()
        return (q, k, v) + run(wp, q, k, v)
    q, k, v, out, lse = forward(x)
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    focus.focus_window_attn_bwd(wp, q, k, v, out, lse, g, focus.alloc_window_bwd_workspace(wp), dq, dk, dv)
    dx = torch.empty_like(x)
    t, dt = x.permute(0, 2, 1, 3), dx.permute(0, 2, 1, 3)
    dw = [torch.empty(d, device="cuda") for _ in range(2)]
    focus.focus_qk_norm_rope_bwd(rp, t[:, :Hq], t[:, Hq:Hq + Hkv], wq, wk, None, turns, dq, dk, focus.alloc_qk_norm_rope_workspace(rp),
                                 dt[:, :Hq], dt[:, Hq:Hq + Hkv], *dw)
    dt[:, Hq + Hkv:] = dv
    f = lambda y: (forward(y)[3].double() * g.double()).sum().item()
    for seed in range(3):
        e = rows(B, n, 8, d, "f32", 8 + seed)
        e /= e.norm()
        assert abs((f(x + 0.01 * e) - f(x - 0.01 * e)) / 0.02 - (dx.double() * e.double()).sum().item()) <= 5e-3
