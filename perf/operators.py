"""What is measured: positions and head norms in front of the attention, and the attention of a sliding window with sinks.

Kinds of case
  rope        focus_rope: queries and keys of a layer rotated by their positions.
  norm_rope   focus_qk_norm_rope: every head of the queries and keys normalised, scaled, then rotated.
  norm_rope_bwd   focus_qk_norm_rope_bwd: the gradients of inputs and of both weights.
  window      focus_window_attn_fwd: key j is seen by row i if j <= i and (i - j < window or j < sinks).
  window_bwd  focus_window_attn_bwd: the gradients of q, k and v.
  window_step focus_window_decode_step_at: one new token for each sequence, over caches that may have wrapped.

Where `own` is false, `run` computes the same from elementary operations in 32 bits (angles in 64) and rounds once.
"""
import math

import torch

own = False

TORCH_DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
ELEM = {"f32": 4, "bf16": 2, "f16": 2}
DEVICE = "cuda"


def listed():
    rope = dict(layout="half", base=10000.0, scaling="none", factor=1.0, original=0, far=0, packed=False)
    window = dict(softcap=0.0, packed=False, lens="")
    return [
        # One token of one sequence, far into its context: launches and latency count.
        dict(rope, kind="rope", name="rope_token", dtype="bf16", B=1, Hq=32, Hkv=8, n=1, d=128, rot=128, far=100000),
        # The other pairing, half of each head rotated, a long prompt whose positions lie past the trained context.
        dict(rope, kind="rope", name="rope_long_partial", dtype="f16", B=1, Hq=32, Hkv=8, n=32768, d=128, rot=64,
             layout="interleaved", base=500000.0, scaling="parts", factor=32.0, original=32768, far=1000000),
        # The new tokens of a batch of generations, each at its own position.
        dict(rope, kind="norm_rope", name="norm_rope_step", dtype="bf16", B=32, Hq=32, Hkv=8, n=1, d=128, rot=128,
             far=30000),
        # A long prompt: q and k taken in place from one projection [B, n, (Hq + 2 Hkv) d].
        dict(rope, kind="norm_rope", name="norm_rope_prefill", dtype="bf16", B=1, Hq=32, Hkv=8, n=32768, d=128, rot=128,
             packed=True),
        # A training batch of a 12-head model.
        dict(rope, kind="norm_rope_bwd", name="norm_rope_bwd_batch8", dtype="bf16", B=8, Hq=12, Hkv=12, n=4096, d=64,
             rot=64),
        # A short prompt kept in 32 bits (evaluation against a reference, small models).
        dict(window, kind="window", name="window_f32_1k", dtype="f32", B=1, Hq=12, Hkv=12, n=1024, d=64, window=128,
             sinks=4),
        # Documents of different lengths end to end in one tensor, 80 components, soft-capped logits.
        dict(window, kind="window", name="window_ragged_f16", dtype="f16", B=7, Hq=15, Hkv=5, n=20011, d=80, window=300,
             sinks=16, softcap=50.0, packed=True, lens="5003 1 7777 130 63 4100 2937"),
        # Grouped queries and a long prompt.
        dict(window, kind="window", name="window_prefill_32k", dtype="bf16", B=1, Hq=32, Hkv=8, n=32768, d=128,
             window=1024, sinks=4),
        # Training: a batch of a 12-head model.
        dict(window, kind="window_bwd", name="window_bwd_batch8_4k", dtype="bf16", B=8, Hq=12, Hkv=12, n=4096, d=64,
             window=256, sinks=4),
        # Training on long sequences with grouped queries.
        dict(window, kind="window_bwd", name="window_bwd_16k", dtype="bf16", B=1, Hq=32, Hkv=8, n=16384, d=128,
             window=1024, sinks=4),
        # Generation for one user.
        dict(window, kind="window_step", name="window_step", dtype="bf16", B=1, Hq=32, Hkv=8, n=1088, d=128, window=1024,
             sinks=4, far=20000),
        # Generation for a batch: caches that have wrapped beside caches that are still filling.
        dict(window, kind="window_step", name="window_step_batch32", dtype="bf16", B=32, Hq=64, Hkv=8, n=4128, d=128,
             window=4096, sinks=4, far=30000),
    ]


# ---------------------------------------------------------------- more cases of the same ranges

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _heads(rng):
    return rng.choice([(12, 12, 64), (16, 16, 64), (32, 8, 128), (64, 8, 128), (16, 4, 256), (40, 8, 96), (15, 5, 80),
                       (32, 32, 128), (24, 8, 128), (14, 2, 64)])


def draw(rng):
    kind = rng.choice(["rope", "norm_rope", "norm_rope_bwd", "window", "window", "window_bwd", "window_bwd", "window_step"])
    Hq, Hkv, d = _heads(rng)
    dtype = rng.choice(["bf16", "bf16", "bf16", "f16", "f32"])
    if kind in ("rope", "norm_rope", "norm_rope_bwd"):
        rows = 32768 * 40 * 128 // ((Hq + Hkv) * d * ELEM[dtype] // 2)
        if kind == "norm_rope_bwd":
            rows //= 4
        n, B = _log_int(rng, 1, rows), rng.choice([1, 1, 2, 4, 8])
        n = max(1, n // B)
        scaling = rng.choice(["none", "none", "linear", "base", "parts", "bands"])
        return dict(kind=kind, dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, n=n, d=d, rot=rng.choice([d, d, d // 2, d // 4]),
                    layout=rng.choice(["half", "half", "interleaved"]), base=rng.choice([10000.0, 500000.0]),
                    scaling=scaling, factor=1.0 if scaling == "none" else rng.choice([2.0, 8.0, 32.0]),
                    original=0 if scaling == "none" else 8192, far=rng.choice([0, 0, _log_int(rng, 1000, 1000000)]),
                    packed=rng.random() < 0.4)
    window, sinks = _log_int(rng, 32, 4096), rng.choice([0, 1, 4, 16, _log_int(rng, 1, 200)])
    softcap = rng.choice([0.0, 0.0, 0.0, 50.0])
    if kind == "window_step":
        B = _log_int(rng, 1, 32)
        if dtype == "f32":
            B = max(1, B // 2)
        return dict(kind=kind, dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, n=window + sinks + rng.choice([0, 1, 32, 500]), d=d,
                    window=window, sinks=sinks, softcap=softcap, packed=False, lens="", far=_log_int(rng, 10, 100000))
    most = 32 * 32768 * 1024 * 128.0 if kind == "window" else 32 * 16384 * 1024 * 128.0
    if dtype == "f32":
        most /= 16
    n, B = _log_int(rng, 1, 32768), rng.choice([1, 1, 2, 4, 8])
    while B > 1 and B * Hq * n * d * float(min(window + sinks, n)) > most:
        B //= 2
    n = max(1, min(n, int(most / (B * Hq * d * min(window + sinks, n)))))
    packed = rng.random() < 0.3
    lens = ""
    if packed:
        cuts = sorted(rng.randint(0, n) for _ in range(B - 1))
        lens = " ".join(str(b - a) for a, b in zip([0] + cuts, cuts + [n]))
    return dict(kind=kind, dtype=dtype, B=B, Hq=Hq, Hkv=Hkv, n=n, d=d, window=window, sinks=sinks, softcap=softcap,
                packed=packed, lens=lens)


# ---------------------------------------------------------------- what a program has in hand before the call

def _generator(seed, salt):
    g = torch.Generator(device=DEVICE)
    g.manual_seed((int(seed) * 1000003 + salt) % (1 << 62))
    return g


def _randn(shape, dt, seed, salt, scale=1.0):
    return (torch.randn(shape, generator=_generator(seed, salt), device=DEVICE) * scale).to(dt)


def _frequencies(case):
    """Turns per position of every pair, and the factor of the rotated components (64 bits, on the host)."""
    r, base, f, L = case["rot"], case["base"], case["factor"], case["original"]
    i = torch.arange(r // 2, dtype=torch.float64)
    if case["scaling"] == "base":
        base = base * f ** (r / (r - 2.0))
    w = base ** (-2.0 * i / r)
    mag = 1.0
    if case["scaling"] == "linear":
        w = w / f
    elif case["scaling"] == "parts":
        at = lambda turns: r * math.log(L / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo, hi = max(math.floor(at(32.0)), 0), min(math.ceil(at(1.0)), r - 1)
        ramp = ((i - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        w = w / f * ramp + w * (1 - ramp)
        mag = 0.1 * math.log(f) + 1.0
    elif case["scaling"] == "bands":
        smooth = ((L * w / (2 * math.pi) - 1.0) / (4.0 - 1.0)).clamp(0, 1)
        w = w / f * (1 - smooth) + w * smooth
    return w / (2 * math.pi), mag


def _lens(case):
    """Lengths of the sequences that lie end to end in one tensor, none if every batch row is a sequence."""
    return [int(x) for x in case["lens"].split()]


def _spans(case):
    if not case["packed"]:
        return None
    rows, first = [], 0
    for x in _lens(case):
        rows.append((first, x))
        first += x
    return torch.tensor(rows, dtype=torch.int32, device=DEVICE)


def _rope_inputs(case, seed):
    B, Hq, Hkv, n, d = (case[x] for x in ("B", "Hq", "Hkv", "n", "d"))
    dt = TORCH_DTYPES[case["dtype"]]
    if case["packed"]:
        qkv = _randn((B, n, Hq + 2 * Hkv, d), dt, seed, 0).permute(0, 2, 1, 3)
        q, k = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv]
    else:
        q, k = _randn((B, Hq, n, d), dt, seed, 1), _randn((B, Hkv, n, d), dt, seed, 2)
    start = torch.randint(0, case["far"] + 1, (B, 1), generator=_generator(seed, 3), device=DEVICE)
    pos = (start + torch.arange(n, device=DEVICE)).to(torch.int32)
    weights = [1.0 + 0.2 * torch.randn((d,), generator=_generator(seed, 4 + x), device=DEVICE) for x in range(2)]
    grads = None
    if case["kind"] == "norm_rope_bwd":
        grads = [_randn((B, Hq, n, d), dt, seed, 6, 0.1), _randn((B, Hkv, n, d), dt, seed, 7, 0.1)]
    return q, k, pos, weights, grads


def _window_inputs(case, seed):
    B, Hq, Hkv, n, d = (case[x] for x in ("B", "Hq", "Hkv", "n", "d"))
    dt = TORCH_DTYPES[case["dtype"]]
    Bt = 1 if case["packed"] else B
    q, k, v = (_randn((Bt, h, n, d), dt, seed, x) for x, h in ((0, Hq), (1, Hkv), (2, Hkv)))
    dout = _randn((Bt, Hq, n, d), dt, seed, 3) if case["kind"] == "window_bwd" else None
    return q, k, v, dout


def _step_inputs(case, seed):
    B, Hq, Hkv, cap, d = (case[x] for x in ("B", "Hq", "Hkv", "n", "d"))
    dt = TORCH_DTYPES[case["dtype"]]
    q, k, v = _randn((B, Hq, d), dt, seed, 0), _randn((B, Hkv, d), dt, seed, 1), _randn((B, Hkv, d), dt, seed, 2)
    kc, vc = _randn((B, Hkv, cap, d), dt, seed, 3), _randn((B, Hkv, cap, d), dt, seed, 4)
    # a quarter of a batch is still within its capacity
    pos = torch.randint(cap, cap + case["far"], (B,), generator=_generator(seed, 5), device=DEVICE)
    young = torch.randint(0, cap, (B,), generator=_generator(seed, 6), device=DEVICE)
    pos = torch.where(torch.arange(B, device=DEVICE) % 4 == 3, young, pos).to(torch.int32)
    return q, k, v, kc, vc, pos


def prepare(case, seed):
    st = dict(case=case)
    if case["kind"] in ("rope", "norm_rope", "norm_rope_bwd"):
        q, k, pos, weights, grads = _rope_inputs(case, seed)
        st.update(q=q, k=k, pos=pos, weights=weights, grads=grads)
        if own:
            from paper_2604_03260_amd import focus
            turns, mag = focus.focus_rope_frequencies(case["rot"], base=case["base"], scaling=case["scaling"],
                                                      factor=case["factor"], original_context=case["original"])
            st.update(turns=turns.to(DEVICE), qo=torch.empty(q.shape, dtype=q.dtype, device=DEVICE),
                      ko=torch.empty(k.shape, dtype=k.dtype, device=DEVICE))
            st["p"] = focus.make_rope_params(case["B"], case["Hq"], case["Hkv"], case["n"], case["d"], case["rot"],
                                             layout=case["layout"], dtype=case["dtype"], magnitude=mag,
                                             q_strides=focus.strides_of(q), k_strides=focus.strides_of(k))
            if grads is not None:
                st.update(ws=focus.alloc_qk_norm_rope_workspace(st["p"]), dw=[torch.empty_like(w) for w in weights])
                if case["packed"]:
                    dqkv = torch.zeros((case["B"], case["n"], case["Hq"] + 2 * case["Hkv"], case["d"]), dtype=q.dtype,
                                       device=DEVICE).permute(0, 2, 1, 3)
                    st.update(qo=dqkv[:, :case["Hq"]], ko=dqkv[:, case["Hq"]:case["Hq"] + case["Hkv"]])
        else:
            turns, mag = _frequencies(case)
            st.update(turns=turns.to(DEVICE), mag=mag)
        return st
    if case["kind"] == "window_step":
        q, k, v, kc, vc, pos = _step_inputs(case, seed)
        st.update(q=q, k=k, v=v, kc=kc, vc=vc, pos=pos)
        if own:
            from paper_2604_03260_amd import focus
            st["p"] = focus.make_window_params(case["B"], case["Hq"], case["Hkv"], case["n"], case["d"], case["window"],
                                               sinks=case["sinks"], dtype=case["dtype"], softcap=case["softcap"])
            st.update(ws=focus.alloc_window_decode_workspace(st["p"]), out=torch.empty_like(q),
                      lse=torch.empty(q.shape[:2], device=DEVICE))
        return st
    q, k, v, dout = _window_inputs(case, seed)
    st.update(q=q, k=k, v=v, dout=dout, spans=_spans(case))
    if own:
        from paper_2604_03260_amd import focus
        st["p"] = focus.make_window_params(case["B"], case["Hq"], case["Hkv"], case["n"], case["d"], case["window"],
                                           sinks=case["sinks"], dtype=case["dtype"], softcap=case["softcap"],
                                           packed=case["packed"], span_max=max(_lens(case), default=0))
        st.update(out=torch.empty_like(q), lse=torch.empty(q.shape[:3], device=DEVICE))
    if dout is not None:
        # the forward pass that a training step has behind it
        if own:
            focus.focus_window_attn_fwd(st["p"], q, k, v, st["out"], st["lse"], spans=st["spans"])
            st.update(ws=focus.alloc_window_bwd_workspace(st["p"]), dq=torch.empty_like(q), dk=torch.empty_like(k),
                      dv=torch.empty_like(v))
        else:
            st["out"], st["lse"] = _window_plain(case, q, k, v)
    return st


# ---------------------------------------------------------------- the plain forms

def _rotate_plain(case, x, pos, turns, mag, inverse):
    """x [B,H,n,d] float32, rotated (mag included)."""
    r = case["rot"]
    t = pos.double()[:, :, None] * turns
    ang = 2 * math.pi * (t - torch.round(t))
    c, s = (torch.cos(ang) * mag).float()[:, None], (torch.sin(ang) * mag).float()[:, None]
    if inverse:
        s = -s
    y = x.clone()
    if case["layout"] == "half":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, b * c + a * s
    return y


def _rope_plain(st):
    case = st["case"]
    outs, dws = [], []
    for x, which in ((st["q"], 0), (st["k"], 1)):
        xf = x.float()
        if case["kind"] == "rope":
            outs.append(_rotate_plain(case, xf, st["pos"], st["turns"], st["mag"], False).to(x.dtype))
            continue
        rstd = torch.rsqrt((xf * xf).mean(-1, keepdim=True) + 1e-6)
        xh, w = xf * rstd, st["weights"][which]
        if case["kind"] == "norm_rope":
            outs.append(_rotate_plain(case, xh * w, st["pos"], st["turns"], st["mag"], False).to(x.dtype))
            continue
        g = _rotate_plain(case, st["grads"][which].float(), st["pos"], st["turns"], st["mag"], True)
        dws.append((g * xh).sum((0, 1, 2), dtype=torch.float64).float())
        g = g * w
        outs.append((rstd * (g - xh * (g * xh).mean(-1, keepdim=True))).to(x.dtype))
    return outs + dws


def _sequences(case):
    """(batch row of the tensors, first row, length) of every sequence."""
    if not case["packed"]:
        return [(b, 0, case["n"]) for b in range(case["B"])]
    rows, first = [], 0
    for x in _lens(case):
        rows.append((0, first, x))
        first += x
    return rows


def _blocks(case, length):
    """Row blocks of a sequence with the keys they can see: (row0, row1, key positions)."""
    step = 512
    for i0 in range(0, length, step):
        i1 = min(i0 + step, length)
        lo = max(0, i0 - case["window"] + 1)
        head = min(case["sinks"], lo)
        yield i0, i1, torch.cat([torch.arange(head, device=DEVICE), torch.arange(lo, i1, device=DEVICE)])


def _logits_plain(case, qb, kb, i0, i1, cols):
    """Masked logits [Hkv,G,rows,keys] (and tanh of the capped ones) of one block."""
    s = torch.matmul(qb, kb.transpose(-1, -2)[:, None]) * (1.0 / math.sqrt(case["d"]))
    t = None
    if case["softcap"]:
        t = torch.tanh(s / case["softcap"])
        s = t * case["softcap"]
    rows = torch.arange(i0, i1, device=DEVICE)[:, None]
    seen = (cols <= rows) & ((rows - cols < case["window"]) | (cols < case["sinks"]))
    return torch.where(seen, s, torch.full_like(s, -math.inf)), t


def _window_plain(case, q, k, v):
    out, lse = torch.empty_like(q), torch.empty(q.shape[:3], device=DEVICE)
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    for b, f, length in _sequences(case):
        for i0, i1, cols in _blocks(case, length):
            qb = q[b, :, f + i0:f + i1].float().reshape(Hkv, Hq // Hkv, i1 - i0, d)
            kb, vb = k[b][:, f + cols].float(), v[b][:, f + cols].float()
            s, _ = _logits_plain(case, qb, kb, i0, i1, cols)
            m = s.amax(-1, keepdim=True)
            p = torch.exp(s - m)
            l = p.sum(-1, keepdim=True)
            out[b, :, f + i0:f + i1] = (torch.matmul(p, vb[:, None]) / l).reshape(Hq, i1 - i0, d).to(q.dtype)
            lse[b, :, f + i0:f + i1] = (m + torch.log(l)).reshape(Hq, i1 - i0)
    return out, lse


def _window_bwd_plain(st):
    case, q, k, v, out, lse, dout = (st[x] for x in ("case", "q", "k", "v", "out", "lse", "dout"))
    Hq, Hkv, d = case["Hq"], case["Hkv"], case["d"]
    dq, dk, dv = torch.empty_like(q), torch.zeros(k.shape, device=DEVICE), torch.zeros(v.shape, device=DEVICE)
    for b, f, length in _sequences(case):
        for i0, i1, cols in _blocks(case, length):
            shape = (Hkv, Hq // Hkv, i1 - i0, d)
            qb, ob, gb = (x[b, :, f + i0:f + i1].float().reshape(shape) for x in (q, out, dout))
            kb, vb = k[b][:, f + cols].float(), v[b][:, f + cols].float()
            s, t = _logits_plain(case, qb, kb, i0, i1, cols)
            p = torch.exp(s - lse[b, :, f + i0:f + i1].reshape(shape[:3])[..., None])
            ds = p * (torch.matmul(gb, vb.transpose(-1, -2)[:, None]) - (gb * ob).sum(-1, keepdim=True))
            if t is not None:
                ds = ds * (1 - t * t)
            ds = ds * (1.0 / math.sqrt(d))
            dq[b, :, f + i0:f + i1] = torch.matmul(ds, kb[:, None]).reshape(Hq, i1 - i0, d).to(q.dtype)
            dk[b].index_add_(1, f + cols, torch.matmul(ds.transpose(-1, -2), qb).sum(1))
            dv[b].index_add_(1, f + cols, torch.matmul(p.transpose(-1, -2), gb).sum(1))
    return [dq, dk.to(k.dtype), dv.to(v.dtype)]


def _slot(case, pos):
    """The cache row of a position: the sinks stay, the others go round."""
    ring = case["n"] - case["sinks"]
    return torch.where(pos < case["n"], pos, case["sinks"] + (pos - case["sinks"]) % ring)


def _step_plain(st):
    case, q, kc, vc, pos = (st[x] for x in ("case", "q", "kc", "vc", "pos"))
    B, Hq, Hkv, d, w, s0 = case["B"], case["Hq"], case["Hkv"], case["d"], case["window"], case["sinks"]
    rows = torch.arange(B, device=DEVICE)
    here = _slot(case, pos.long())
    kc[rows, :, here], vc[rows, :, here] = st["k"], st["v"]
    at = torch.cat([torch.arange(s0, device=DEVICE).expand(B, -1),
                    pos.long()[:, None] - w + 1 + torch.arange(w, device=DEVICE)], 1)
    first = torch.arange(s0 + w, device=DEVICE) < s0
    seen = (at >= 0) & (at <= pos[:, None]) & (first | (at >= s0))
    slot = _slot(case, at.clamp(min=0))
    kb, vb = kc[rows[:, None], :, slot].float(), vc[rows[:, None], :, slot].float()      # [B,keys,Hkv,d]
    qb = q.float().reshape(B, Hkv, Hq // Hkv, d)
    s = torch.matmul(qb, kb.permute(0, 2, 3, 1)) * (1.0 / math.sqrt(d))
    if case["softcap"]:
        s = torch.tanh(s / case["softcap"]) * case["softcap"]
    s = torch.where(seen[:, None, None], s, torch.full_like(s, -math.inf))
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - m)
    l = p.sum(-1, keepdim=True)
    out = (torch.matmul(p, vb.permute(0, 2, 1, 3)) / l).reshape(B, Hq, d).to(q.dtype)
    return [out, (m + torch.log(l)).reshape(B, Hq), kc, vc]


# ---------------------------------------------------------------- one pass

def run(st):
    case = st["case"]
    kind = case["kind"]
    if not own:
        if kind in ("rope", "norm_rope", "norm_rope_bwd"):
            return _rope_plain(st)
        if kind == "window":
            return list(_window_plain(case, st["q"], st["k"], st["v"]))
        return _window_bwd_plain(st) if kind == "window_bwd" else _step_plain(st)
    from paper_2604_03260_amd import focus
    p = st["p"]
    if kind == "rope":
        focus.focus_rope(p, st["q"], st["k"], st["pos"], st["turns"], st["qo"], st["ko"])
        return [st["qo"], st["ko"]]
    if kind == "norm_rope":
        focus.focus_qk_norm_rope(p, st["q"], st["k"], st["weights"][0], st["weights"][1], st["pos"], st["turns"],
                                 st["qo"], st["ko"])
        return [st["qo"], st["ko"]]
    if kind == "norm_rope_bwd":
        focus.focus_qk_norm_rope_bwd(p, st["q"], st["k"], st["weights"][0], st["weights"][1], st["pos"], st["turns"],
                                     st["grads"][0], st["grads"][1], st["ws"], st["qo"], st["ko"], st["dw"][0],
                                     st["dw"][1])
        return [st["qo"], st["ko"]] + st["dw"]
    if kind == "window":
        focus.focus_window_attn_fwd(p, st["q"], st["k"], st["v"], st["out"], st["lse"], spans=st["spans"])
        return [st["out"], st["lse"]]
    if kind == "window_bwd":
        focus.focus_window_attn_bwd(p, st["q"], st["k"], st["v"], st["out"], st["lse"], st["dout"], st["ws"], st["dq"],
                                    st["dk"], st["dv"], spans=st["spans"])
        return [st["dq"], st["dk"], st["dv"]]
    focus.focus_window_decode_step_at(p, st["pos"], st["q"], st["k"], st["v"], st["kc"], st["vc"], st["ws"], st["out"],
                                      st["lse"])
    return [st["out"], st["lse"], st["kc"], st["vc"]]


# ---------------------------------------------------------------- what a pass cannot do without

def _pairs(case, length):
    """Pairs that a sequence of that length attends."""
    w, s0 = case["window"], case["sinks"]
    m = min(length, w)
    total = m * (m + 1) // 2 + (length - m) * w
    for j in range(min(s0, max(0, length - w))):           # rows i >= j + w see sink j beside their window
        total += length - w - j
    return total


def work(case):
    B, Hq, Hkv, n, d, e = case["B"], case["Hq"], case["Hkv"], case["n"], case["d"], ELEM[case["dtype"]]
    if case["kind"] in ("rope", "norm_rope", "norm_rope_bwd"):
        elems = B * n * (Hq + Hkv) * d
        rotated = elems // d * case["rot"]
        if case["kind"] == "rope":
            return {"bytes": 2 * elems * e + 4 * B * n, "flops": 3 * rotated}
        if case["kind"] == "norm_rope":
            return {"bytes": 2 * elems * e + 4 * B * n + 8 * d, "flops": 4 * elems + 3 * rotated}
        return {"bytes": 3 * elems * e + 4 * B * n + 16 * d, "flops": 11 * elems + 3 * rotated}
    if case["kind"] == "window_step":
        keys = min(case["window"] + case["sinks"], n)
        rows = B * Hkv * keys * d
        return {"bytes": 2 * rows * e + (2 * Hq + 4 * Hkv) * B * d * e + 4 * B * Hq, "flops": 4 * B * Hq * keys * d}
    pairs = Hq * sum(_pairs(case, length) for _, _, length in _sequences(case))
    rows = (1 if case["packed"] else B) * n
    if case["kind"] == "window":
        return {"bytes": rows * ((2 * Hq + 2 * Hkv) * d * e + 4 * Hq), "flops": 4 * d * pairs}
    return {"bytes": rows * ((4 * Hq + 4 * Hkv) * d * e + 4 * Hq), "flops": 10 * d * pairs}


# ---------------------------------------------------------------- the definition in 64 bits

def _exact_angles(case, pos):
    """exp(i angle), complex128 [B,1,n,rot/2], times the factor of the rotated components."""
    r, f, L = case["rot"], case["factor"], float(case["original"])
    base = case["base"] * (f ** (r / (r - 2.0)) if case["scaling"] == "base" else 1.0)
    omega, mag = [], 1.0
    for i in range(r // 2):
        w = math.pow(base, -2.0 * i / r)
        turns_in_context = L * w / (2 * math.pi)
        if case["scaling"] == "linear":
            w /= f
        elif case["scaling"] == "parts":
            lo = max(math.floor(r / 2 * math.log(L / (64 * math.pi)) / math.log(base)), 0)
            hi = min(math.ceil(r / 2 * math.log(L / (2 * math.pi)) / math.log(base)), r - 1)
            keep = 1.0 - min(1.0, max(0.0, (i - lo) / max(hi - lo, 0.001)))
            w = w * keep + w / f * (1.0 - keep)
            mag = 1.0 + math.log(f) / 10.0
        elif case["scaling"] == "bands":
            if turns_in_context < 1.0:
                w /= f
            elif turns_in_context < 4.0:
                keep = (turns_in_context - 1.0) / 3.0
                w = (1.0 - keep) * w / f + keep * w
        omega.append(w)
    ang = pos.double()[..., None] * torch.tensor(omega, dtype=torch.float64, device=DEVICE)
    return torch.polar(torch.full_like(ang, mag), ang)[:, None]


def _exact_rotate(case, x, z):
    r = case["rot"]
    rot = x[..., :r]
    pairs = rot.unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else rot.unflatten(-1, (r // 2, 2))
    y = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
    y = y.transpose(-1, -2).flatten(-2) if case["layout"] == "half" else y.flatten(-2)
    return torch.cat([y, x[..., r:]], -1)


def _exact_window(case, q, k, v, dout):
    outs = {"out": torch.empty(q.shape, dtype=torch.float64, device=DEVICE),
            "lse": torch.empty(q.shape[:3], dtype=torch.float64, device=DEVICE)}
    grads = [torch.zeros(x.shape, dtype=torch.float64, device=DEVICE) for x in (q, k, v)] if dout is not None else None
    G, w, s0, cap = case["Hq"] // case["Hkv"], case["window"], case["sinks"], case["softcap"]
    for b, f, length in _sequences(case):
        for h in range(case["Hkv"]):
            heads = slice(h * G, (h + 1) * G)
            for i0 in range(0, length, 1024):
                i1 = min(length, i0 + 1024)
                a0 = max(0, i0 - w + 1)
                near = slice(f + a0, f + i1)
                far = slice(f, f + min(s0, a0))
                qd = q[b, heads, f + i0:f + i1].double().requires_grad_(dout is not None)
                kd = torch.cat([k[b, h, far], k[b, h, near]]).double().requires_grad_(dout is not None)
                vd = torch.cat([v[b, h, far], v[b, h, near]]).double().requires_grad_(dout is not None)
                key = torch.cat([torch.arange(far.stop - far.start, device=DEVICE), torch.arange(a0, i1, device=DEVICE)])
                ahead = torch.arange(i0, i1, device=DEVICE)[:, None] - key[None, :]
                hidden = (ahead < 0) | ((ahead >= w) & (key[None, :] >= s0))
                logit = (qd.reshape(-1, case["d"]) @ kd.T).reshape(G, i1 - i0, -1) / math.sqrt(case["d"])
                if cap:
                    logit = cap * torch.tanh(logit / cap)
                logit = logit.masked_fill(hidden, -math.inf)
                total = torch.logsumexp(logit, -1)
                o = (torch.exp(logit - total[..., None]).reshape(G * (i1 - i0), -1) @ vd).reshape(G, i1 - i0, -1)
                outs["out"][b, heads, f + i0:f + i1] = o.detach()
                outs["lse"][b, heads, f + i0:f + i1] = total.detach()
                if dout is None:
                    continue
                gq, gk, gv = torch.autograd.grad(o, (qd, kd, vd), dout[b, heads, f + i0:f + i1].double())
                nfar = far.stop - far.start
                grads[0][b, heads, f + i0:f + i1] = gq
                for g, x in ((grads[1], gk), (grads[2], gv)):
                    g[b, h, far] += x[:nfar]
                    g[b, h, near] += x[nfar:]
    return [outs["out"], outs["lse"]] if grads is None else grads


def _exact_step(case, q, k, v, kc, vc, pos):
    s0, w, cap = case["sinks"], case["window"], case["softcap"]
    out = torch.empty(q.shape, dtype=torch.float64, device=DEVICE)
    lse = torch.empty(q.shape[:2], dtype=torch.float64, device=DEVICE)
    kc, vc = kc.clone(), vc.clone()
    for b, p in enumerate(pos.tolist()):
        row = lambda x: x if x < case["n"] else s0 + (x - s0) % (case["n"] - s0)
        kc[b, :, row(p)], vc[b, :, row(p)] = k[b], v[b]
        seen = [row(x) for x in range(p + 1) if x < s0] + [row(x) for x in range(max(s0, p - w + 1), p + 1)] \
            if p < 2 * (s0 + w) else [row(x) for x in range(s0)] + [row(x) for x in range(p - w + 1, p + 1)]
        idx = torch.tensor(seen, device=DEVICE)
        kd, vd = kc[b][:, idx].double(), vc[b][:, idx].double()
        logit = torch.matmul(q[b].double().reshape(case["Hkv"], -1, case["d"]), kd.transpose(1, 2).contiguous()) / math.sqrt(case["d"])
        if cap:
            logit = cap * torch.tanh(logit / cap)
        out[b] = torch.matmul(torch.softmax(logit, -1), vd).reshape(case["Hq"], case["d"])
        lse[b] = torch.logsumexp(logit, -1).reshape(-1)
    return [out, lse, kc.double(), vc.double()]


def exact(case, seed):
    if case["kind"] in ("rope", "norm_rope", "norm_rope_bwd"):
        q, k, pos, weights, grads = _rope_inputs(case, seed)
        z = _exact_angles(case, pos)
        outs, dws = [], []
        for i, x in enumerate((q, k)):
            x = x.double()
            if case["kind"] == "rope":
                outs.append(_exact_rotate(case, x, z))
                continue
            w = weights[i].double()
            if case["kind"] == "norm_rope":
                outs.append(_exact_rotate(case, x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + 1e-6) * w, z))
                continue
            x.requires_grad_(True)
            w.requires_grad_(True)
            y = _exact_rotate(case, x / torch.sqrt((x * x).sum(-1, keepdim=True) / case["d"] + 1e-6) * w, z)
            gx, gw = torch.autograd.grad(y, (x, w), grads[i].double())
            outs.append(gx)
            dws.append(gw)
        return outs + dws
    if case["kind"] == "window_step":
        return _exact_step(case, *_step_inputs(case, seed))
    return _exact_window(case, *_window_inputs(case, seed))
