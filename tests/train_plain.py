"""The training operators in 64 bits, from their formulas, and bounds on how far a 32-bit kernel may be from them.

Bounds are first-order rounding bounds: a sum of m terms in fp32 in any order is off by at most about m 2^-24 times the sum of
the terms' magnitudes (2^-23 where an adder truncates, as tensor cores may), a value rounded to a type by its unit roundoff."""
import math

import torch

ROUND = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}     # unit roundoff
TINY = {torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -149}   # half the smallest subnormal


def embed(table, ids, scale, pad):
    t = table.double()
    V = t.shape[0]
    ok = (ids >= 0) & (ids < V)
    out = t[ids.clamp(0, V - 1)] * scale
    out = torch.where(ok[..., None], out, float("nan"))
    return torch.where((ids == pad)[..., None] & (pad >= 0), torch.zeros_like(out), out)


def embed_backward(dout, ids, V, scale, pad):
    """(gradient, sum of magnitudes, largest number of terms of a sum)"""
    D = dout.shape[-1]
    ids, d = ids.reshape(-1), dout.reshape(-1, D).double()
    live = (ids >= 0) & (ids < V)
    if pad >= 0:
        live &= ids != pad
    g = torch.zeros(V, D, dtype=torch.float64, device=d.device).index_add_(0, ids[live], d[live] * scale)
    a = torch.zeros(V, D, dtype=torch.float64, device=d.device).index_add_(0, ids[live], d[live].abs() * abs(scale))
    m = int(torch.bincount(ids[live], minlength=1).max()) if int(live.sum()) else 0
    return g, a, m


A, B = math.sqrt(2.0 / math.pi), 0.044715


def gelu(v):
    return 0.5 * v * (1.0 + torch.tanh(A * (v + B * v ** 3)))


def gelu_slope(v):
    t = torch.tanh(A * (v + B * v ** 3))
    return 0.5 * (1.0 + t) + 0.5 * v * (1.0 - t * t) * A * (1.0 + 3.0 * B * v ** 2)


def save8(x):
    """q and scales by the operator's fp32 definition, one IEEE operation at a time, on the CPU."""
    x = x.detach().cpu().float()
    n, d = x.shape
    groups = -(-d // 128)
    p = torch.zeros(n, groups * 128)
    p[:, :d] = x
    p = p.view(n, groups, 128)
    a = p.abs().amax(2)                      # NaN where a group holds one
    live = (a > 2.0 ** -100) & torch.isfinite(a)
    inv = torch.where(live, torch.full_like(a, 127.0) / a, torch.zeros_like(a))
    third = torch.full((), 1.0) / torch.full((), 127.0)
    scale = torch.where(live, a * third, torch.where(torch.isfinite(a), torch.zeros_like(a), torch.full_like(a, float("nan"))))
    q = torch.where(live[..., None], (p * inv[..., None]).round(), torch.zeros_like(p))
    return q.view(n, groups * 128)[:, :d].to(torch.int8), scale


def load8(q, scales):
    n, d = q.shape
    return (q.float() * scales.repeat_interleave(128, 1)[:, :d])


def vocab_loss(h, w, t, ignore, c):
    """loss, lse, and the labelled rows with their logits"""
    V = w.shape[0]
    N = len(t)
    ok = (t != ignore) & (t >= 0) & (t < V)
    rows = ok.nonzero()[:, 0]
    nan, zero = torch.full((N,), float("nan"), dtype=torch.float64, device=h.device), torch.zeros(N, dtype=torch.float64, device=h.device)
    loss = torch.where(ok | (t == ignore), zero, nan)
    lse = loss.clone()
    l = c * (h[rows].double() @ w.double().t())
    lse[rows] = torch.logsumexp(l, 1)
    loss[rows] = lse[rows] - l.gather(1, t[rows][:, None])[:, 0]
    return loss, lse, rows, l


def vocab_logit_error(h, w, rows, c):
    """What a logit may be off by: D products summed with a truncating adder, twice over for the adder's own width; and the scale."""
    D = h.shape[1]
    s = (h[rows].double().abs() @ w.double().abs().t()).amax(1) if len(rows) else torch.zeros(0, dtype=torch.float64, device=h.device)
    return abs(c) * s * (D + 8) * 2.0 ** -22


def vocab_backward(h, w, t, ignore, c, dloss):
    """dh, dw, and g of the labelled rows"""
    _, lse, rows, l = vocab_loss(h, w, t, ignore, c)
    g = torch.exp(l - lse[rows][:, None])
    g[torch.arange(len(rows), device=h.device), t[rows]] -= 1.0
    g *= dloss[rows].double()[:, None] * c
    dh = torch.zeros(h.shape, dtype=torch.float64, device=h.device)
    dh[rows] = g @ w.double()
    return dh, g.t() @ h[rows].double(), g, rows
