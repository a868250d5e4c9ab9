"""The attention of a sliding window with sinks and its gradients in 64 bits, from the definition, with error bounds of the kernels.

Bounds, per result.  u = half a step of the storage type relative to the value (bf16 2^-8, fp16 2^-11, fp32 2^-24), e = 2^-24.
  A logit is d exact products (fp32: rounded ones) summed in 32 bits, scaled, soft-capped: off by at most
  EL = (d + 8) e |scale| sum|q k| + 4 e softcap (tanh within 2 ulp) + 4 e |logit| (the exponent in units of log 2, and its reference).
  A probability is off by EP = EL + 4 e relative, and rounded once for the product (u); IEEE halves drop what is below 2^-31 of the row's largest.
  out: u |out| + sum p |v| (u + 2 EP + (keys + 8) e) + 2^-31 sum |v| (the last for halves).
  Exponentials below 2^-126 = 1.2e-38 become zero (v_exp_f32 makes no subnormal numbers): a term that met magnitudes of up to 10^6 is then off by
  1.2e-32, 10^4 such terms by 1.2e-28: FLUSH = 2e-28 absolute for everything that is a sum over probabilities.
  lse: max EL + (keys + 8) e + 2 e |lse|.
  In the gradient P comes from the kernel's own lse: EP + (its error); dS = P (dout.v - delta) is off by
  ES = |dS| (EP' + u) + P (d + 4) e sum|dout v| + P sum|dout| (error of out, which is rounded, + (d + 4) e |out|), 2^-25 more for halves
  (subnormal), and each gradient is the sum of these times the magnitudes it meets, (terms + 8) e of its terms' magnitudes, and u of itself.
"""
import math

import torch

HALF_STEP = {"f32": 2.0 ** -24, "bf16": 2.0 ** -8, "f16": 2.0 ** -11}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
E = 2.0 ** -24
FLUSH = 2e-28


def mask(length, window, sinks, device="cuda"):
    i = torch.arange(length, device=device)
    dist = i[:, None] - i[None, :]
    return (dist >= 0) & ((dist < window) | (i[None, :] < sinks))


def reference(q, k, v, window, sinks, scale, softcap, dtype, dout=None):
    """One sequence: q [Hq,len,d], k, v [Hkv,len,d] -> dict of results in 64 bits, and their bounds under name + '_tol'."""
    Hq, n, d = q.shape
    Hkv = k.shape[0]
    G = Hq // Hkv
    u = HALF_STEP[dtype]
    half = dtype == "f16"
    q, k, v = q.double(), k.double(), v.double()
    ke, ve = k.repeat_interleave(G, 0), v.repeat_interleave(G, 0)
    see = mask(n, window, sinks)
    keys = see.sum(-1).double()[None, :, None]
    raw = torch.matmul(q, ke.transpose(1, 2).contiguous()) * scale
    el = (d + 8) * E * scale * torch.matmul(q.abs(), ke.abs().transpose(1, 2).contiguous())
    x = softcap * torch.tanh(raw / softcap) if softcap else raw
    el = el + 4 * E * x.abs() + 4 * E * softcap
    el = torch.where(see, el, torch.zeros_like(el)).amax(-1, keepdim=True)
    x = x.masked_fill(~see, -math.inf)
    lse = torch.logsumexp(x, -1)
    p = torch.exp(x - lse[..., None])
    r = {"out": torch.matmul(p, ve), "lse": lse}
    ep = el + 4 * E
    r["out_tol"] = u * r["out"].abs() + torch.matmul(p, ve.abs()) * ((u if dtype != "f32" else 0) + 2 * ep + (keys + 8) * E)
    if half:
        r["out_tol"] = r["out_tol"] + 2.0 ** -31 * torch.matmul(see.double(), ve.abs()) + 2.0 ** -25
    r["lse_tol"] = (el + (keys + 8) * E)[..., 0] + 2 * E * lse.abs()
    if dout is None:
        return r
    g = dout.double()
    ep2 = (2 * ep + (keys + 8) * E + 4 * E * lse.abs()[..., None])
    dp = torch.matmul(g, ve.transpose(1, 2).contiguous())
    delta = (g * r["out"]).sum(-1, keepdim=True)
    damp = 1 - torch.tanh(raw / softcap) ** 2 if softcap else 1.0
    ds = p * (dp - delta) * damp
    w = u if dtype != "f32" else 0
    es = ds.abs() * (ep2 + w) + p * ((d + 4) * E * torch.matmul(g.abs(), ve.abs().transpose(1, 2).contiguous())
                                    + (g.abs() * (r["out_tol"] + (d + 4) * E * r["out"].abs())).sum(-1, keepdim=True))
    if softcap:                                        # 1 - tanh^2 from a tanh within 4 e of an argument off by el / softcap
        es = es + p * (dp - delta).abs() * (2 * el / softcap + 16 * E)
    if half:
        es = es + 2.0 ** -25 * see
    rows = float(G * n)
    fold = lambda t: t.reshape(Hkv, G, n, -1).sum(1)
    r["dq"] = torch.matmul(ds, ke) * scale
    r["dq_tol"] = u * r["dq"].abs() + scale * torch.matmul(es + (keys + 8) * E * ds.abs(), ke.abs())
    dst, est, pt = (t.transpose(1, 2).contiguous() for t in (ds, es, p))
    r["dk"] = fold(torch.matmul(dst, q)) * scale
    r["dk_tol"] = u * r["dk"].abs() + scale * fold(torch.matmul(est + (rows + 8) * E * dst.abs(), q.abs()))
    r["dv"] = fold(torch.matmul(pt, g))
    pe = (p * (ep2 + w + (rows + 8) * E)).transpose(1, 2).contiguous()
    if half:
        pe = pe + 2.0 ** -25 * see.T
    r["dv_tol"] = u * r["dv"].abs() + fold(torch.matmul(pe, g.abs()))
    if half:
        for x in ("dq", "dk", "dv"):
            r[x + "_tol"] = r[x + "_tol"] + 2.0 ** -25
    return r


def check(got, ref, name):
    err = (got.double() - ref[name]).abs()
    bad = ~(err <= ref[name + "_tol"] + FLUSH)
    assert not bad.any(), "%s: %d of %d, worst %.3g of its bound" % (
        name, int(bad.sum()), bad.numel(), float((err / ref[name + "_tol"]).nan_to_num(nan=math.inf).max()))
