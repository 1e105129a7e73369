"""The gated delta rule and its gradients, token by token in 64 bits, and how large what enters each result is.

Sizes, for each row and head, by norms over the head's columns and the largest of them over all steps (Cauchy-Schwarz), with C = 32
steps of a chunk, or T if that is less:
  o       scale |q| (|S| + C |u|)                 dq  scale |do| (|S| + C |u|)
  dv      |R|                                     dk  |R| |u| + |S| |z| + C (scale |do| |u| |q| + 2 |z| |u|)
  dbeta   |R| |e|      state  |S|   dstate0  |R|  dlog_decay  |R| |S| + C^2 / 2 (scale |do| |u| |q| + |z| |u|)
(u = beta e, z the gradient of v, keys of unit length.)

Tolerances.  A step makes a rounding of at most (dk + 2 C) 2^-24 of its size (sums of dk products, of up to C of the chunk's
steps, and of C in the substitution).  A step maps an error in the state to one that is no larger (|I - beta k k^T| <= 1 for strengths
up to 2) and is decayed besides, so errors add up over the memory's length L at most: the state is off by n 2^-24 of the largest
state, n = (dk + dv + 2 C) (C + L), R alike, and what both enter by twice that.  bf16 results: what enters the last products
as two terms leaves out 2^-16 of each factor, three factors' worth at most, and the result is rounded to 8 bits.
"""
import math

import torch

CHUNK = 32


def oracle(x, scale=None, do=None, dstate=None):
    """x: q, k [T,N,Hk,dk], v [T,N,H,dv], log_decay, beta [T,N,H], done or None, state0 or None.  Results, and their sizes."""
    q, v = x["q"], x["v"]
    T, N, Hk, dk = q.shape
    H, dv = v.shape[2:]
    f64 = dict(dtype=torch.float64, device=q.device)
    C = min(CHUNK, T)
    scale = dk ** -0.5 if scale is None else scale
    rep = lambda a: a.double().repeat_interleave(H // Hk, 2)
    q, k, v, beta = rep(x["q"]), rep(x["k"]), v.double(), x["beta"].double()
    begin = (x["done"] != 0)[..., None].expand(T, N, H) if x.get("done") is not None else torch.zeros(T, N, H, dtype=torch.bool, device=q.device)
    begin = begin | (x["log_decay"].double() * 1.4426950408889634 < -126)
    a = torch.where(begin, 0.0, x["log_decay"].double().exp())
    s = torch.zeros(N, H, dk, dv, **f64) if x.get("state0") is None else x["state0"].double()
    o, before, es = torch.zeros(T, N, H, dv, **f64), [], []
    norm = lambda m, n=1: m.flatten(-n).norm(dim=-1)
    top = dict(s=norm(s, 2), r=torch.zeros(N, H, **f64), u=torch.zeros(N, H, **f64), e=torch.zeros(N, H, **f64), z=torch.zeros(N, H, **f64))

    def seen(name, m, n):
        top[name] = torch.maximum(top[name], norm(m, n))

    for t in range(T):
        s = torch.where(begin[t][..., None, None], 0.0, a[t][..., None, None] * s)
        e = v[t] - (s * k[t][..., :, None]).sum(-2)
        before.append(s)
        es.append(e)
        u = beta[t][..., None] * e
        s = s + k[t][..., :, None] * u[..., None, :]
        o[t] = scale * (s * q[t][..., :, None]).sum(-2)
        seen("s", s, 2), seen("u", u, 1), seen("e", e, 1)
    big = lambda m: (norm(m) if T else torch.zeros(1, N, H, **f64)).amax(0)  # [N, H]
    per = lambda m: m[:, :, None]
    if do is None:
        nq = norm(q)
        return dict(o=o, state=s), dict(o=(abs(scale) * nq * (top["s"] + C * top["u"]))[..., None], state=top["s"][..., None, None])
    do = do.double()
    r = torch.zeros_like(s) if dstate is None else dstate.double()
    top["r"] = norm(r, 2)
    g = {n: [None] * T for n in ("dq", "dk", "dv", "dlog_decay", "dbeta")}
    for t in reversed(range(T)):
        u = beta[t][..., None] * es[t]
        after = before[t] + k[t][..., :, None] * u[..., None, :]
        g["dq"][t] = scale * (after * do[t][..., None, :]).sum(-1)
        r = r + scale * q[t][..., :, None] * do[t][..., None, :]
        du = (r * k[t][..., :, None]).sum(-2)
        seen("r", r, 2)
        z = beta[t][..., None] * du
        seen("z", z, 1)
        g["dv"][t] = z
        g["dbeta"][t] = (du * es[t]).sum(-1)
        g["dk"][t] = (r * u[..., None, :]).sum(-1) - (before[t] * z[..., None, :]).sum(-1)
        r = r - k[t][..., :, None] * z[..., None, :]
        g["dlog_decay"][t] = torch.where(begin[t], 0.0, (r * before[t]).sum((-1, -2)))
        r = torch.where(begin[t][..., None, None], 0.0, a[t][..., None, None] * r)
        seen("r", r, 2)
    empty = dict(dq=q, dk=k, dv=v, dlog_decay=beta, dbeta=beta)
    g = {n: torch.stack(m) if T else torch.zeros_like(empty[n]) for n, m in g.items()}
    share = lambda m: m.unflatten(2, (Hk, H // Hk)).sum(3)
    g["dq"], g["dk"], g["dstate0"] = share(g["dq"]), share(g["dk"]), r
    sc, S, R, u, e, z, D, Q = abs(scale), top["s"], top["r"], top["u"], top["e"], top["z"], big(do), big(q)
    heads = lambda m: m.unflatten(-1, (Hk, H // Hk)).sum(-1)
    size = dict(dq=heads(sc * D * (S + C * u))[..., None], dk=heads(R * u + S * z + C * (sc * D * u * Q + 2 * z * u))[..., None], dv=R[..., None], dbeta=R * e,
                dlog_decay=R * S + C * C / 2 * (sc * D * u * Q + z * u), dstate0=R[..., None, None])
    return g, size


def tolerance(name, y, size, dk, dv, length, bf16, T):
    C = min(CHUNK, T)
    n = 2 * (dk + dv + 2 * C) * (C + min(length, T))
    tol = n * 2.0 ** -24 * size
    if bf16 and name in ("o", "dq", "dk", "dv"):
        tol = (tol + 3 * 2.0 ** -16 * size) * (1 + 2.0 ** -8) + 2.0 ** -8 * y.abs()
    return tol + 1e-37


def check(got, want, size, dk, dv, length, bf16, T, part=None):
    """part: steps that are looked at (of results that have steps)."""
    for name, y in want.items():
        x, tol = got[name].double(), tolerance(name, y, size[name], dk, dv, length, bf16, T)
        assert x.shape == y.shape, name
        tol = tol.expand_as(y)
        if part is not None and "state" not in name:
            x, y, tol = x[part], y[part], tol[part]
        bad = torch.isfinite(y) != torch.isfinite(x)
        assert not bad.any(), "%s: %d of other finiteness" % (name, bad.sum())
        fine = torch.isfinite(y)
        over = ((x - y).abs()[fine] / tol[fine]).max().item() if fine.any() else 0.0
        assert over <= 1.0, "%s: %.2f of the tolerance" % (name, over)


def make(T, N, H, Hk, dk, dv, dtype, p_done=0.1, seed=0, memory=16.0, device="cuda"):
    """Inputs whose decays keep a memory of at most `memory` steps; their gradients' inputs do and dstate."""
    g = torch.Generator(device=device).manual_seed(seed)
    dt = torch.bfloat16 if dtype == "bf16" else dtype if isinstance(dtype, torch.dtype) else torch.float32
    r = lambda *s: torch.randn(s, generator=g, device=device)
    unit = lambda a: a / a.norm(dim=-1, keepdim=True).clamp(min=1e-20)
    x = dict(q=r(T, N, Hk, dk).to(dt), k=unit(r(T, N, Hk, dk)).to(dt), v=r(T, N, H, dv).to(dt), log_decay=-(1.0 / memory + r(T, N, H).square() / memory),
             beta=torch.sigmoid(r(T, N, H)), done=(torch.rand(T, N, generator=g, device=device) < p_done).byte(), state0=0.3 * r(N, H, dk, dv))
    return x, r(T, N, H, dv).to(dt), 0.3 * r(N, H, dk, dv)
