"""Attention over packed sequences in 64 bits, and how far results may be from it.

``reference`` gives outputs, gradients and for each a bound, element by element, counted from the roundings that a kernel cannot
avoid or chooses to make.  u: half a step of the storage type (bf16 2^-8, fp32 2^-24); f = 2^-23: a step of fp32, allowed for every
addition of an fp32 sum (a matrix instruction may round down; half a step would be rounding to nearest).

    score     e_s = f (d + 2) scale sum |q||k| + 2 f |s|            (largest of a row: it moves weights and sum alike)
    weight    relative: 2 e_s + 4 f; and u_w where it is rounded for its product (bf16: 2^-8, fp32: kept)
    a         (weight + f (lk + 2)) sum p|v|, + u |a|
    lse       e_s + f (lk + 2) + 2 f |lse|
    dP, D     f (d + 2) sum |da||v|,  (f (d + 2) + u) sum |da||a|    (a is stored in between)
    dS        p (weight |dP - D| + e_dP + e_D), + u_w |dS|
    dq, dk    scale sum e_dS |k|, + f n scale sum |dS||k|, + u |dq|;   dv as a
"""
import math

import torch

F = 2.0 ** -23
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def spans(offsets, lengths):
    out = []
    for i in range(len(offsets) - 1):
        n = offsets[i + 1] - offsets[i]
        out.append((offsets[i], n if lengths is None else min(lengths[i], n)))
    return out


def reference(q, k, v, da, q_spans, k_spans, scale=None):
    """q, da: [tokens, kv, group, d]; k, v: [tokens, kv, d]; lists of (first row, length).  {name: (value, bound)} with zeros (and
    bound 0) in rows of no sequence; da None: forward only."""
    u = HALF_STEP[q.dtype]
    u_w = u if q.dtype == torch.bfloat16 else 0.0
    tq, kv, r, d = q.shape
    scale = scale or 1.0 / math.sqrt(d)
    z = lambda *shape: (torch.zeros(shape, dtype=torch.float64, device=q.device), torch.zeros(shape, dtype=torch.float64, device=q.device))   # noqa: E731
    out = {"a": z(*q.shape), "lse": z(kv * r, tq)}
    if da is not None:
        out.update(dq=z(*q.shape), dk=z(*k.shape), dv=z(*k.shape))
    for (q0, lq), (k0, lk) in zip(q_spans, k_spans):
        qs, ks = slice(q0, q0 + lq), slice(k0, k0 + lk)
        if lq == 0:
            continue
        seen = torch.ones(lq, lk, dtype=torch.bool, device=q.device).tril(lk - lq)
        some = seen.any(-1, keepdim=True) if lk else torch.zeros(lq, 1, dtype=torch.bool, device=q.device)
        for j in range(kv):
            K, V = k[ks, j].double(), v[ks, j].double()
            for g in range(r):
                Q = q[qs, j, g].double()
                s = torch.where(seen, Q @ K.T * scale, -math.inf)
                lse = torch.logsumexp(s, -1, keepdim=True) if lk else torch.full((lq, 1), -math.inf, dtype=torch.float64, device=q.device)
                p = torch.where(seen, torch.exp(s - lse), 0.0)
                e_s = torch.where(seen, F * ((d + 2) * scale * (Q.abs() @ K.abs().T) + 2 * s.abs()), 0.0)
                e_s = e_s.amax(-1, keepdim=True) if lk else torch.zeros_like(lse)
                w = 2 * e_s + 4 * F
                a, pv = p @ V, p @ V.abs()
                put = lambda name, at, value, bound: (out[name][0][at].add_(value), out[name][1][at].add_(bound))   # noqa: E731
                put("a", (qs, j, g), a, (w + u_w + F * (lk + 2)) * pv + u * a.abs())
                put("lse", (j * r + g, qs), lse[:, 0], torch.where(some, e_s + F * (lk + 2) + 2 * F * lse.abs(), 0.0)[:, 0])
                if da is None:
                    continue
                dA = da[qs, j, g].double()
                dP, D = dA @ V.T, (dA * a).sum(-1, keepdim=True)
                e = F * (d + 2) * (dA.abs() @ V.abs().T) + (F * (d + 2) + u) * (dA.abs() * a.abs()).sum(-1, keepdim=True)
                dS = p * (dP - D)
                e_dS = p * (w * (dP - D).abs() + e) + u_w * dS.abs()
                dq = scale * dS @ K
                put("dq", (qs, j, g), dq, scale * (e_dS + F * lk * dS.abs()) @ K.abs() + u * dq.abs())
                put("dk", (ks, j), scale * dS.T @ Q, scale * (e_dS + F * r * lq * dS.abs()).T @ Q.abs())
                put("dv", (ks, j), p.T @ dA, ((w + u_w + F * r * lq) * p).T @ dA.abs())
    if da is not None:
        for name in ("dk", "dv"):
            value, bound = out[name]
            out[name] = (value, bound + u * value.abs())
    return out


def assert_within(got, want, what):
    value, bound = want
    if not got.numel():
        return
    got = got.double()
    same = (got == value) | (torch.isnan(got) & torch.isnan(value))
    off = torch.where(same, 0.0, (got - value).abs() - bound * (1 + 1e-6))
    assert not torch.isnan(off).any(), f"{what}: NaN where there should be none, or none where there should be"
    worst = int(off.argmax())
    assert off.max() <= 0, f"{what}: element {worst} is {got.flatten()[worst]} and not {value.flatten()[worst]} +- {bound.flatten()[worst]}"
