"""Frequencies and refusals of the rotary calls: host code only."""
import ctypes
import math

import pytest
import torch

from paper_2604_03260_amd import focus

vp = ctypes.c_void_p


def literal(r, base, scaling, f, L, fast, slow):
    out = []
    for i in range(r // 2):
        b = base * f ** (r / (r - 2)) if scaling == "base" else base
        w = b ** (-2 * i / r)
        if scaling == "linear":
            w = w / f
        if scaling == "parts":
            at = lambda turns: r / 2 * math.log(L / (2 * math.pi * turns)) / math.log(b)
            lo, hi = max(0, math.floor(at(fast))), min(r - 1, math.ceil(at(slow)))
            x = min(1, max(0, (i - lo) / max(hi - lo, 0.001)))
            w = (1 - x) * w + x * w / f
        if scaling == "bands":
            turns = L * w / (2 * math.pi)
            x = 0 if turns > fast else 1 if turns < slow else (fast - turns) / (fast - slow)
            w = (1 - x) * w + x * w / f
        out.append(w / (2 * math.pi))
    return out


@pytest.mark.parametrize("scaling,fast,slow", [("none", 0, 0), ("linear", 0, 0), ("base", 0, 0), ("parts", 32, 1), ("bands", 4, 1), ("bands", 8, 2)])
@pytest.mark.parametrize("r", [4, 20, 64, 128, 256])
def test_frequencies(scaling, fast, slow, r):
    turns, mag = focus.focus_rope_frequencies(r, base=10000.0, scaling=scaling, factor=8.0, original_context=4096, fast=fast, slow=slow)
    want = torch.tensor(literal(r, 10000.0, scaling, 1.0 if scaling == "none" else 8.0, 4096, fast, slow), dtype=torch.float64)
    assert torch.allclose(turns, want, rtol=1e-13, atol=0)
    assert mag == pytest.approx(0.1 * math.log(8.0) + 1 if scaling == "parts" else 1.0, rel=1e-7)
    if scaling in ("parts", "bands") and (fast, slow) != (8, 2):
        assert torch.equal(turns, focus.focus_rope_frequencies(r, scaling=scaling, factor=8.0, original_context=4096)[0])
    if scaling == "base" and r > 2:                    # the slowest pair is slowed by the factor, the fastest not at all
        plain = focus.focus_rope_frequencies(r)[0]
        assert turns[0] == plain[0] and turns[-1].item() == pytest.approx(plain[-1].item() / 8.0, rel=1e-12)


@pytest.mark.parametrize("kw", [dict(rot_dim=0), dict(rot_dim=7), dict(rot_dim=258), dict(base=1.0), dict(base=float("nan")),
                                dict(scaling="linear", factor=0.5), dict(scaling="linear", factor=float("inf")),
                                dict(scaling="parts", factor=2.0), dict(scaling="bands", factor=2.0, original_context=8192, fast=1, slow=2),
                                dict(scaling="base", factor=2.0, rot_dim=2)])
def test_frequencies_refuse(kw):
    args = dict(rot_dim=64)
    args.update(kw)
    with pytest.raises(focus.FocusError) as e:
        focus.focus_rope_frequencies(**args)
    assert e.value.status == focus.FOCUS_EINVAL


def call(fn="focus_rope", ptrs=None, ws=None, **kw):
    args = dict(B=1, Hq=4, Hkv=2, n=16, d=64, rot_dim=64)
    args.update(kw)
    p = focus.make_rope_params(**args)
    lib = focus.load_library()
    P = dict(q=0x10000, k=0x20000, qw=0x30000, kw=0x40000, pos=0x50000, turns=0x60000, gq=0x70000, gk=0x80000, oq=0x90000, ok=0xa0000,
             dqw=0xb0000, dkw=0xc0000, ws=0xd0000)
    P.update(ptrs or {})
    v = {x: vp(y) for x, y in P.items()}
    if fn == "focus_rope":
        st = lib.focus_rope(ctypes.byref(p), 0, v["q"], v["k"], v["pos"], v["turns"], v["oq"], v["ok"], vp(0))
    elif fn == "focus_qk_norm_rope":
        st = lib.focus_qk_norm_rope(ctypes.byref(p), v["q"], v["k"], v["qw"], v["kw"], v["pos"], v["turns"], v["oq"], v["ok"], vp(0))
    else:
        st = lib.focus_qk_norm_rope_bwd(ctypes.byref(p), v["q"], v["k"], v["qw"], v["kw"], v["pos"], v["turns"], v["gq"], v["gk"], v["ws"],
                                        0 if ws is None else ws, v["oq"], v["ok"], v["dqw"], v["dkw"], vp(0))
    return st, focus.focus_last_error()


BAD_PARAMS = [(dict(B=0), focus.FOCUS_EINVAL), (dict(Hq=0), focus.FOCUS_EINVAL), (dict(n=0), focus.FOCUS_EINVAL),
              (dict(Hkv=-1), focus.FOCUS_EINVAL), (dict(d=72), focus.FOCUS_EUNSUPPORTED), (dict(rot_dim=66), focus.FOCUS_EINVAL),
              (dict(rot_dim=7), focus.FOCUS_EINVAL), (dict(rot_dim=0), focus.FOCUS_EINVAL), (dict(n=1 << 25), focus.FOCUS_EUNSUPPORTED),
              (dict(eps=-1.0), focus.FOCUS_EINVAL), (dict(magnitude=float("nan")), focus.FOCUS_EINVAL),
              (dict(q_strides=(4096, 1024, 65)), focus.FOCUS_EINVAL), (dict(qo_strides=(4096, -1024, 64)), focus.FOCUS_EINVAL),
              (dict(B=65535, Hq=2), focus.FOCUS_EUNSUPPORTED)]


@pytest.mark.parametrize("kw,want", BAD_PARAMS)
def test_params_refused(kw, want):
    st, msg = call(**kw)
    assert st == want, msg


@pytest.mark.parametrize("fn,ptrs,kw", [
    ("focus_rope", dict(q=0), {}), ("focus_rope", dict(ok=0), {}), ("focus_rope", dict(turns=0), {}), ("focus_rope", dict(q=0x10008), {}),
    ("focus_rope", dict(turns=0x60004), {}), ("focus_rope", dict(ok=0x90000), {}), ("focus_rope", dict(oq=0x20000), {}),
    ("focus_rope", {}, dict(Hkv=0)), ("focus_rope", dict(oq=0x10000), dict(q_strides=(4096, 64, 256))),
    ("focus_qk_norm_rope", dict(qw=0), {}), ("focus_qk_norm_rope", dict(kw=0), {}), ("focus_qk_norm_rope", dict(kw=0x40002), {}),
    ("focus_qk_norm_rope_bwd", dict(gq=0), {}), ("focus_qk_norm_rope_bwd", dict(dkw=0), {}), ("focus_qk_norm_rope_bwd", dict(ws=0), {}),
    ("focus_qk_norm_rope_bwd", dict(oq=0x80000), {}), ("focus_qk_norm_rope_bwd", dict(oq=0x70000), dict(q_strides=(4096, 64, 256))),
])
def test_pointers_refused(fn, ptrs, kw):
    st, msg = call(fn, ptrs, ws=1 << 30, **kw)
    assert st == focus.FOCUS_EINVAL, msg


def test_workspace_of_the_gradient():
    need = focus.focus_qk_norm_rope_workspace_size(focus.make_rope_params(1, 4, 2, 16, 64, 64))
    assert need > 0
    assert call("focus_qk_norm_rope_bwd", ws=0)[0] == focus.FOCUS_EWORKSPACE
    assert call("focus_qk_norm_rope_bwd", dict(ws=0xd0010), ws=need)[0] == focus.FOCUS_EWORKSPACE


def test_null_params():
    lib = focus.load_library()
    assert lib.focus_rope(None, 0, vp(0), vp(0), vp(0), vp(0), vp(0), vp(0), vp(0)) == focus.FOCUS_EINVAL
    assert lib.focus_rope_frequencies(None, vp(0), None) == focus.FOCUS_EINVAL
    assert lib.focus_qk_norm_rope_workspace_size(None, None) == focus.FOCUS_EINVAL
