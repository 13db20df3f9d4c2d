"""Attention and its gradients in 64 bits on the host, from the definition in q2d.h."""
import math

import torch


def seen(Lq, Lk, causal=True, window=0, documents=None, prefix=0):
    """[Lq, Lk] truth table of one sequence."""
    p = torch.arange(Lk - Lq, Lk)[:, None]
    j = torch.arange(Lk)[None, :]
    ok = torch.ones((Lq, Lk), dtype=torch.bool)
    if causal:
        ok &= j <= p
    if window:
        ok &= (p - j).abs() < window
    ok |= j < prefix
    if documents is not None:
        d = documents.to(torch.int64)
        dq = torch.where(p >= 0, d[p.clamp(min=0)], torch.full_like(p, -1))
        ok &= (dq == d[None, :]) & (dq >= 0)
    return ok


def attention(q, k, v, dout=None, scale=None, causal=True, window=0, softcap=0.0, slopes=None, documents=None, prefix=None):
    """out, lse and (with dout) dq, dk, dv of [batch, length, heads, dim] tensors."""
    q, k, v = (t.detach().cpu().double() for t in (q, k, v))
    B, Lq, Hq, D = q.shape
    Lk, Hkv = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    out, lse = torch.zeros_like(q), torch.full((B, Hq, Lq), -math.inf, dtype=torch.float64)
    grads = None
    if dout is not None:
        dout = dout.detach().cpu().double()
        grads = [torch.zeros_like(t) for t in (q, k, v)]
    dist = (torch.arange(Lk - Lq, Lk)[:, None] - torch.arange(Lk)[None, :]).abs().double()
    for b in range(B):
        ok = seen(Lq, Lk, causal, window, None if documents is None else documents[b].cpu(),
                  0 if prefix is None else int(prefix[b]))
        some = ok.any(1)
        for h in range(Hq):
            g = h // (Hq // Hkv)
            # what is not seen has no influence, whatever it holds: zeros in its place
            live_k, live_q = ok.any(0), some
            qh = torch.where(live_q[:, None], q[b, :, h], 0.0)
            kh, vh = (torch.where(live_k[:, None], t[b, :, g], 0.0) for t in (k, v))
            x = scale * (qh @ kh.T)
            th = torch.tanh(x / softcap) if softcap else None
            s = softcap * th if softcap else x
            if slopes is not None:
                s = s - float(slopes[h]) * dist
            s = torch.where(ok, s, -math.inf)
            m = torch.where(some, s.amax(1), 0.0)[:, None]
            e = torch.where(ok, torch.exp(s - m), 0.0)
            z = e.sum(1, keepdim=True)
            P = e / torch.where(some[:, None], z, 1.0)
            out[b, :, h] = _masked(P, vh, ok)
            lse[b, h] = torch.where(some, (m + torch.log(z))[:, 0], -math.inf)
            if dout is None:
                continue
            do = torch.where(live_q[:, None], dout[b, :, h], 0.0)
            dP = torch.where(ok, do @ vh.T, 0.0)
            delta = torch.where(some, (P * dP).sum(1), 0.0)[:, None]
            dS = torch.where(ok, P * (dP - delta), 0.0)
            if softcap:
                dS = torch.where(ok, dS * (1 - th * th), 0.0)
            grads[0][b, :, h] = scale * _masked(dS, kh, ok)
            grads[1][b, :, g] += scale * _masked(dS.T, qh, ok.T)
            grads[2][b, :, g] += _masked(P.T, do, ok.T)
    return (out, lse) if dout is None else (out, lse) + tuple(grads)


def _masked(w, x, ok):
    """w @ x over the pairs in ok alone (x may hold infinities and NaN elsewhere)."""
    if torch.isfinite(x).all() and torch.isfinite(w).all():
        return w @ x
    r = torch.zeros((w.shape[0], x.shape[1]), dtype=w.dtype)
    for i in range(w.shape[0]):
        r[i] = w[i][ok[i]] @ x[ok[i]] if ok[i].any() else 0.0
    return r
