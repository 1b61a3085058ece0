"""Softmax attention of one sequence in 64 bits on the CPU, from its definition, with the
largest error that the library's arithmetic allows each result.

u: half a step of the dtype (eps / 2), the error of one rounding relative to the value.
Weights, P and dS are rounded once (u), results once (u); products are exact in fp32 and their
sums carry at most n 2^-24 of the sum of |terms|; an exponential of a score that is off by e is
off by e relative, besides 2^-21 of its own.  fp16 numbers below 2^-14 are rounded to steps of
2^-24: `tiny` for results, and the scaled copies of P (2^15) and dS (their bound X below 2^15)
bring that to 2^-40 and X 2^-38."""
import math

import torch

EPS32 = 2.0 ** -24


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def visible(m, n, causal, window):
    i = torch.arange(m).unsqueeze(1) + (n - m)
    j = torch.arange(n).unsqueeze(0)
    see = torch.ones(m, n, dtype=torch.bool)
    if causal:
        see &= j <= i
        if window:
            see &= j > i - window
    return see


def one(q, k, v, scale, causal=False, window=0, dout=None, see=None):
    """q: m x Hq x D, k: n x Hkv x D, v: n x Hkv x C (any device, 16-bit).  Returns
    {name: (value, bound)} for out, lse (Hq x m) and, with dout, dq, dk, dv."""
    dt = q.dtype
    u, tiny = half_step(dt), (2.0 ** -24 if dt == torch.float16 else 0.0)
    m, Hq, D = q.shape
    n, Hkv, C = v.shape
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    if see is None:
        see = visible(m, n, causal, window)
    out, bout = torch.zeros(m, Hq, C).double(), torch.zeros(m, Hq, C).double()
    lse, blse = torch.full((Hq, m), -math.inf).double(), torch.zeros(Hq, m).double()
    res = {"out": (out, bout), "lse": (lse, blse)}
    if dout is not None:
        g = dout.detach().cpu().double()
        for name, t in (("dq", q), ("dk", k), ("dv", v)):
            res[name] = (torch.zeros_like(t), torch.zeros_like(t))
        X = 2 * g.nan_to_num(0, 0, 0).norm(dim=-1).max().item() * v.nan_to_num(0, 0, 0).norm(dim=-1).max().item() if m and n else 0.0
    if m == 0 or n == 0:
        return res
    some = see.any(1)
    for h in range(Hq):
        hk = h // (Hq // Hkv)
        qh, kh, vh = q[:, h], k[:, hk], v[:, hk]
        x = (qh @ kh.t()).mul(scale).masked_fill(~see, -math.inf)
        z = torch.logsumexp(x, 1)
        lse[h] = z
        p = torch.exp(x - z.masked_fill(~some, 0.0).unsqueeze(1)).masked_fill(~see, 0.0)
        out[:, h] = p @ vh
        # scores: their sums, the factor, and the exponent's own rounding
        size = (qh.abs() @ kh.abs().t()).mul(abs(scale)).masked_fill(~see, 0.0)
        es = (size.amax(1) * (D + 3) + x.masked_fill(~see, 0.0).abs().amax(1) * 4) * EPS32 + 2.0 ** -21
        blse[h] = 2 * es + z.masked_fill(~some, 0.0).abs() * 4 * EPS32 + n * EPS32
        ew = (2 * es + n * EPS32).unsqueeze(1)
        A = p @ vh.abs()
        bout[:, h] = (u + ew + n * EPS32) * A + u * out[:, h].abs() * (1 + 2 * u) + tiny + n * 2.0 ** -45 * vh.abs().amax()
        if dout is None:
            continue
        gh = g[:, h]
        ep = es.unsqueeze(1) + blse[h].unsqueeze(1)
        dp = gh @ vh.t()
        delta = (gh * out[:, h]).sum(1, keepdim=True)
        ds = p * (dp - delta)
        # the backward pass takes the rounded out
        edelta = (gh.abs() * bout[:, h]).sum(1, keepdim=True) + C * EPS32 * (gh.abs() * out[:, h].abs()).sum(1, keepdim=True)
        edp = (C + 3) * EPS32 * (gh.abs() @ vh.abs().t())
        eds = (u + ep) * ds.abs() + p * (1 + ep) * (edp + edelta) + (X * 2.0 ** -38 if tiny else 0.0) * see
        res["dq"][0][:, h] = scale * (ds @ kh)
        res["dq"][1][:, h] = abs(scale) * ((eds + n * EPS32 * ds.abs()) @ kh.abs())
        res["dk"][0][:, hk] += scale * (ds.t() @ qh)
        res["dk"][1][:, hk] += abs(scale) * ((eds + m * Hq * EPS32 * ds.abs()).t() @ qh.abs())
        res["dv"][0][:, hk] += p.t() @ gh
        res["dv"][1][:, hk] += ((u + ep + m * Hq * EPS32) * p + (2.0 ** -40 if tiny else 0.0) * see).t() @ gh.abs()
    if dout is not None:
        for name in ("dq", "dk", "dv"):
            val, bound = res[name]
            bound += u * (val.abs() + bound) + tiny
    return res


def check(name, got, want, bound):
    got, want = got.detach().cpu().double(), want.reshape(got.shape)
    bound = bound.reshape(got.shape)
    fine = torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want)), "%s: NaN in other places" % name
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)]), "%s: infinities" % name
    over = (got - want).abs()[fine] > bound[fine] + 1e-300
    if over.any():
        err = ((got - want).abs()[fine] / (bound[fine] + 1e-300))
        raise AssertionError("%s: %d of %d over the bound, worst %.3g times" % (name, int(over.sum()), over.numel(), err.max()))
