"""Refusals and sizes of the window calls: host code only."""
import ctypes

import pytest

from paper_2604_03260_amd import focus

vp = ctypes.c_void_p
BASE = dict(B=1, Hq=4, Hkv=2, n=256, d=64, window=16, sinks=2)
PTR = {x: 0x10000 * (i + 1) for i, x in enumerate(("q", "k", "v", "out", "lse", "dout", "spans", "ws", "dq", "dk", "dv", "kc", "vc", "pos"))}


def call(fn, ptrs=None, ws=1 << 40, capacity=64, **kw):
    p = focus.make_window_params(**{**BASE, **kw})
    lib = focus.load_library()
    v = {x: vp(y) for x, y in {**PTR, "spans": 0, **(ptrs or {})}.items()}
    r = ctypes.byref(p)
    if fn == "fwd":
        st = lib.focus_window_attn_fwd(r, v["q"], v["k"], v["v"], v["spans"], v["out"], v["lse"], vp(0))
    elif fn == "bwd":
        st = lib.focus_window_attn_bwd(r, v["q"], v["k"], v["v"], v["out"], v["lse"], v["dout"], v["spans"], v["ws"], ws, v["dq"], v["dk"],
                                       v["dv"], vp(0))
    elif fn == "fill":
        st = lib.focus_window_cache_fill(r, capacity, v["k"], v["v"], v["spans"], v["kc"], v["vc"], vp(0))
    else:
        st = lib.focus_window_decode_step_at(r, v["pos"], v["q"], v["k"], v["v"], v["kc"], v["vc"], v["ws"], ws, v["out"], v["lse"], vp(0))
    return st, focus.focus_last_error()


@pytest.mark.parametrize("fn", ["fwd", "bwd", "fill", "step"])
@pytest.mark.parametrize("kw,want", [
    (dict(B=0), focus.FOCUS_EINVAL), (dict(Hq=5), focus.FOCUS_EINVAL), (dict(Hkv=0), focus.FOCUS_EINVAL), (dict(n=0), focus.FOCUS_EINVAL),
    (dict(window=0), focus.FOCUS_EINVAL), (dict(sinks=-1), focus.FOCUS_EINVAL), (dict(d=72), focus.FOCUS_EUNSUPPORTED),
    (dict(n=1 << 25), focus.FOCUS_EUNSUPPORTED), (dict(Hq=512, Hkv=2), focus.FOCUS_EUNSUPPORTED), (dict(B=40000), focus.FOCUS_EUNSUPPORTED),
    (dict(scale=-1.0), focus.FOCUS_EINVAL), (dict(softcap=float("nan")), focus.FOCUS_EINVAL), (dict(span_max=257), focus.FOCUS_EINVAL),
    (dict(span_max=-1), focus.FOCUS_EINVAL), (dict(q_strides=(16384, 4096, 65)), focus.FOCUS_EINVAL),
    (dict(kv_strides=(-8, 4096, 64)), focus.FOCUS_EINVAL), (dict(o_strides=(64, 64, 1 << 24)), focus.FOCUS_EUNSUPPORTED)])
def test_params_refused(fn, kw, want):
    st, msg = call(fn, **kw)
    assert st == want, msg


@pytest.mark.parametrize("fn,ptrs", [
    (fn, {x: y}) for fn, names in (("fwd", "q k v out"), ("bwd", "q k v out dout dq dk dv"), ("fill", "k v kc vc"), ("step", "q k v kc vc out"))
    for x in names.split() for y in (0, 0x10008)] + [
    ("fwd", dict(out=PTR["q"])), ("fwd", dict(lse=0x10002)), ("fwd", dict(spans=0x10004)), ("bwd", dict(lse=0)), ("bwd", dict(ws=0)),
    ("bwd", dict(dq=PTR["q"])), ("bwd", dict(dk=PTR["v"])), ("bwd", dict(dv=PTR["dout"])), ("bwd", dict(dk=PTR["dv"])), ("bwd", dict(dq=PTR["dv"])),
    ("fill", dict(kc=PTR["k"])), ("fill", dict(kc=PTR["vc"])), ("step", dict(pos=0)), ("step", dict(pos=0x10002)), ("step", dict(out=PTR["q"])),
    ("step", dict(kc=PTR["vc"])), ("step", dict(ws=0))])
def test_pointers_refused(fn, ptrs):
    st, msg = call(fn, ptrs)
    assert st == focus.FOCUS_EINVAL, msg


def test_packed_sequences_need_spans():
    for fn in ("fwd", "bwd", "fill"):
        st, msg = call(fn, packed=True, B=3)
        assert st == focus.FOCUS_EINVAL and "spans" in msg


def test_caches_of_a_step_are_contiguous():
    assert call("step", packed=True)[0] == focus.FOCUS_EUNSUPPORTED
    assert call("step", q_strides=(16384, 4096, 64))[0] == focus.FOCUS_EUNSUPPORTED


def test_a_prompt_has_to_fit_caches_that_cannot_go_round():
    assert call("fill", n=256, window=60, sinks=5, capacity=64)[0] == focus.FOCUS_EINVAL
    assert call("fill", capacity=0)[0] == focus.FOCUS_EINVAL
    assert call("fill", n=256, window=300, sinks=2 ** 31 - 1, capacity=255)[0] == focus.FOCUS_EINVAL


@pytest.mark.parametrize("fn,size", [("bwd", "focus_window_bwd_workspace_size"), ("step", "focus_window_decode_workspace_size")])
def test_workspaces(fn, size):
    p = focus.make_window_params(**BASE)
    need = ctypes.c_size_t(0)
    lib = focus.load_library()
    assert getattr(lib, size)(ctypes.byref(p), ctypes.byref(need)) == focus.FOCUS_OK and need.value > 0 and need.value % 256 == 0
    assert call(fn, dict(ws=0x10010))[0] == focus.FOCUS_EWORKSPACE
    if fn == "bwd":
        assert call(fn, ws=255)[0] == focus.FOCUS_EWORKSPACE
    assert getattr(lib, size)(None, ctypes.byref(need)) == focus.FOCUS_EINVAL
    assert getattr(lib, size)(ctypes.byref(p), None) == focus.FOCUS_EINVAL
