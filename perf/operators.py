"""The training operators, as cases that can be timed and compared: what a micro-batch of a language model computes at its
vocabulary (lookup, loss, their gradients) and what it saves of its activations.

`run` with `own` false is the plain form of each operator in elementary torch operations, in 32 bits; with `own` true it is
the calls a user makes of ``paper_2306_10598_b200.api``.  `exact` is the operator's definition in 64 bits.

  vocab_loss   loss_n = log sum_v exp(l_nv) - l_{n,t_n},  l = c h W^T, over the rows that carry a label; its gradients
  embed        out_n = s table[id_n]; its gradient, the sum of the output gradients of each token
  gelu_save8   y = gelu(x), x kept as 8-bit integers with a scale for each 128 of a row; the backward pass from those
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
NO_LABEL = -100
PAD = 0
GROUP = 128


def listed():
    return [
        # scoring a handful of tokens with a trained head: one pass over the weight, latency counts
        {"name": "loss score 8 tokens", "op": "loss", "train": False, "N": 8, "V": 32000, "D": 1024, "keep": 1.0, "dtype": "bf16"},
        # held-out loss of a batch, no gradient
        {"name": "loss score 4096 f16", "op": "loss", "train": False, "N": 4096, "V": 32000, "D": 1024, "keep": 1.0, "dtype": "f16"},
        # a toy model's step: odd row length, odd vocabulary, some rows without a label
        {"name": "loss step odd sizes", "op": "loss", "train": True, "N": 251, "V": 5003, "D": 129, "keep": 0.9, "dtype": "f16"},
        # masked-token training: about 15 % of the positions carry a label
        {"name": "loss step 15% labelled", "op": "loss", "train": True, "N": 16384, "V": 32768, "D": 1024, "keep": 0.15, "dtype": "bf16"},
        # next-token training of a whole micro-batch with a large vocabulary
        {"name": "loss step 8192 x 65536", "op": "loss", "train": True, "N": 8192, "V": 65536, "D": 1024, "keep": 1.0, "dtype": "bf16"},
        # the lookup of a single short sequence
        {"name": "embed 16 tokens", "op": "embed", "grad": False, "N": 16, "V": 32000, "D": 1024, "dtype": "bf16", "accumulate": False},
        # the lookup of a large micro-batch
        {"name": "embed 65536 tokens", "op": "embed", "grad": False, "N": 65536, "V": 50021, "D": 1024, "dtype": "bf16", "accumulate": False},
        # gradient accumulation: a micro-batch's gradient added to the 32-bit sum of those before it
        {"name": "embed grad accumulated", "op": "embed", "grad": True, "N": 16384, "V": 32768, "D": 1024, "dtype": "bf16", "accumulate": True},
        # a gradient by itself, odd sizes, 32-bit training
        {"name": "embed grad odd f32", "op": "embed", "grad": True, "N": 5001, "V": 30011, "D": 771, "dtype": "f32", "accumulate": False},
        # a toy layer with an odd width
        {"name": "gelu odd f16", "op": "gelu", "N": 67, "D": 1001, "dtype": "f16"},
        # the inner width of a layer, a usual micro-batch
        {"name": "gelu 4096 x 4096", "op": "gelu", "N": 4096, "D": 4096, "dtype": "bf16"},
        # a large one
        {"name": "gelu 16384 x 8192", "op": "gelu", "N": 16384, "D": 8192, "dtype": "bf16"},
    ]


def _log_int(rng, lo, hi):
    """A whole number spread evenly over the logarithm of [lo, hi]; every other one is odd, the others multiples of 8 where there is room."""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    n = n | 1 if rng.random() < 0.5 else max(8, n // 8 * 8)
    return min(max(n, lo), hi)


def draw(rng):
    op = rng.choice(("loss", "loss", "embed", "embed", "gelu"))
    if op == "loss":
        train = rng.random() < 0.6
        c = {"op": op, "train": train, "N": _log_int(rng, 1, 8192), "V": _log_int(rng, 1000, 65536), "D": _log_int(rng, 64, 1024),
             "keep": rng.choice((1.0, 1.0, 0.85, 0.15)), "dtype": rng.choice(("bf16", "bf16", "f16"))}
    elif op == "embed":
        grad = rng.random() < 0.6
        c = {"op": op, "grad": grad, "N": _log_int(rng, 1, 65536), "V": _log_int(rng, 1000, 65536), "D": _log_int(rng, 64, 1024),
             "dtype": rng.choice(("bf16", "bf16", "f16", "f32")), "accumulate": grad and rng.random() < 0.5}
    else:
        c = {"op": op, "N": _log_int(rng, 1, 16384), "D": _log_int(rng, 64, 8192), "dtype": rng.choice(("bf16", "bf16", "f16", "f32"))}
    return c


def _labelled(case):
    return max(1, round(case["keep"] * case["N"]))


def _tokens(n, V, g):
    """Tokens whose frequency falls like 1 / rank, as words' does."""
    u = torch.rand(n, generator=g, device="cuda", dtype=torch.float64)
    return (torch.exp(u * math.log(V + 1)).long() - 1).clamp_(0, V - 1)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt, N, D = DTYPES[case["dtype"]], case["N"], case["D"]
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    s = {"case": case}
    if case["op"] == "loss":
        V = case["V"]
        # logits of a model part-way through training: the label stands out by 0 to 10
        weight = normal(V, D) * (1.0 / math.sqrt(D))
        targets = _tokens(N, V, g)
        lift = torch.rand(N, 1, generator=g, device="cuda") * 10.0
        hidden = normal(N, D) + lift * weight[targets]
        order = torch.randperm(N, generator=g, device="cuda")
        targets[order[_labelled(case):]] = NO_LABEL
        s.update(hidden=hidden.to(dt), weight=weight.to(dt), targets=targets)
        if case["train"]:
            # the mean over labelled rows, as the loss of a micro-batch is reduced; rows differ a little (weights of sequences)
            s["dloss"] = (0.75 + 0.5 * torch.rand(N, generator=g, device="cuda")) / _labelled(case)
    elif case["op"] == "embed":
        V = case["V"]
        ids = _tokens(N, V, g)
        ids[torch.rand(N, generator=g, device="cuda") < 0.05] = PAD
        s.update(ids=ids, scale=math.sqrt(D))
        if case["grad"]:
            s["dout"] = (normal(N, D) * 1e-2).to(dt)
            if case["accumulate"]:
                s["dtable"] = normal(V, D) * 1e-2
        else:
            s["table"] = (normal(V, D) * (1.0 / math.sqrt(D))).to(dt)
    else:
        x = normal(N, D)
        x *= torch.where(torch.rand(1, D, generator=g, device="cuda") < 0.01, 8.0, 1.0)  # a few channels run large
        s.update(x=x.to(dt), dy=(normal(N, D) * 1e-2).to(dt))
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _plain_loss(s, train):
    h, w, t = s["hidden"], s["weight"], s["targets"]
    rows = (t != NO_LABEL).nonzero()[:, 0]
    hf, wf, tr = h[rows].float(), w.float(), t[rows]
    logits = hf @ wf.t()
    top = logits.amax(1, keepdim=True)
    lse_r = top[:, 0] + torch.exp(logits - top).sum(1).log()
    at = torch.arange(len(rows), device=h.device)
    loss = torch.zeros(len(t), device=h.device)
    lse = torch.zeros(len(t), device=h.device)
    loss[rows] = lse_r - logits[at, tr]
    lse[rows] = lse_r
    if not train:
        return loss, lse
    grad = torch.exp(logits - lse_r[:, None])
    grad[at, tr] -= 1.0
    grad *= s["dloss"][rows][:, None]
    dhidden = torch.zeros_like(h)
    dhidden[rows] = (grad @ wf).to(h.dtype)
    return loss, lse, dhidden, (grad.t() @ hf).to(w.dtype)


def _plain_embed(s):
    ids, scale = s["ids"], s["scale"]
    live = (ids != PAD)[:, None]
    if "table" in s:
        return torch.where(live, s["table"][ids].float() * scale, 0.0).to(s["table"].dtype)
    d = torch.where(live, s["dout"].float() * scale, 0.0)
    if "dtable" in s:
        return s["dtable"].index_add_(0, ids, d)
    return torch.zeros(s["case"]["V"], d.shape[1], device=d.device).index_add_(0, ids, d)


A = math.sqrt(2.0 / math.pi)
B = 0.044715


def _plain_gelu(x, dy):
    n, d = x.shape
    xf = x.float()
    y = xf / (1.0 + torch.exp(-2.0 * A * (xf + B * xf * xf * xf)))
    xp = torch.cat([xf, torch.zeros(n, -d % GROUP, device=x.device)], 1).view(n, -1, GROUP)
    top = xp.abs().amax(2, keepdim=True)
    inv = torch.where(top > 2.0 ** -100, torch.full_like(top, 127.0) / top, 0.0)
    scale = torch.where(top > 2.0 ** -100, top * (1.0 / 127.0), 0.0)
    saved = (xp * inv).round().to(torch.int8)
    v = (saved.float() * scale).view(n, -1)[:, :d]
    sig = 1.0 / (1.0 + torch.exp(-2.0 * A * (v + B * v * v * v)))
    dx = dy.float() * (sig + v * sig * (1.0 - sig) * (2.0 * A) * (1.0 + 3.0 * B * v * v))
    return y.to(x.dtype), dx.to(x.dtype), (v * sig).to(x.dtype)


def run(s):
    case = s["case"]
    if not own:
        if case["op"] == "loss":
            return _plain_loss(s, case["train"])
        return _plain_embed(s) if case["op"] == "embed" else _plain_gelu(s["x"], s["dy"])
    from paper_2306_10598_b200 import api
    if case["op"] == "loss":
        loss, lse = api.vocab_loss(s["hidden"], s["weight"], s["targets"], ignore_index=NO_LABEL)
        if not case["train"]:
            return loss, lse
        dhidden, dweight = api.vocab_loss_backward(s["hidden"], s["weight"], s["targets"], lse, s["dloss"], ignore_index=NO_LABEL)
        return loss, lse, dhidden, dweight
    if case["op"] == "embed":
        if not case["grad"]:
            return api.embed(s["table"], s["ids"], scale=s["scale"], pad_id=PAD)
        if case["accumulate"]:
            return api.embed_backward(s["dout"], s["ids"], case["V"], scale=s["scale"], pad_id=PAD, dtable=s["dtable"], accumulate=True)
        return api.embed_backward(s["dout"], s["ids"], case["V"], scale=s["scale"], pad_id=PAD, dtype=torch.float32)
    y, saved, scales = api.gelu_save8(s["x"])
    dx, y_again = api.gelu_save8_backward(s["dy"], saved, scales, want_y=True)
    return y, dx, y_again


def work(case):
    N, D, e = case["N"], case["D"], 4 if case["dtype"] == "f32" else 2
    if case["op"] == "loss":
        L, V = _labelled(case), case["V"]
        read = (L * D + V * D) * e + 8 * N
        if not case["train"]:
            return {"bytes": read + 8 * N, "flops": 2 * L * V * D}
        return {"bytes": read + 4 * N + 8 * N + (N * D + V * D) * e, "flops": 6 * L * V * D}
    if case["op"] == "embed":
        V = case["V"]
        # tokens that fall like 1 / rank: how many different ones N draws are expected to hold
        ranks = torch.arange(1, V + 1, dtype=torch.float64)
        different = float((1.0 - (1.0 - torch.log1p(1.0 / ranks) / math.log(V + 1)) ** N).sum())
        if not case["grad"]:
            return {"bytes": 8 * N + (different + N) * D * e, "flops": N * D}
        table = 2 * different * D * 4 if case["accumulate"] else V * D * 4
        return {"bytes": 8 * N + N * D * e + table, "flops": 2 * N * D}
    # forward: x in, y, 8 bits and scales out; backward: dy, 8 bits and scales in, dx and y out
    return {"bytes": N * D * (5 * e + 2) + 8 * N * (-(-D // GROUP)), "flops": 30 * N * D}


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "loss":
        t = s["targets"]
        N, V, D = case["N"], case["V"], case["D"]
        w = s["weight"].double()
        loss, lse = torch.zeros(N, dtype=torch.float64, device="cuda"), torch.zeros(N, dtype=torch.float64, device="cuda")
        dh, dw = torch.zeros(N, D, dtype=torch.float64, device="cuda"), torch.zeros(V, D, dtype=torch.float64, device="cuda")
        for lo in range(0, N, 2048):
            part = slice(lo, lo + 2048)
            has = t[part] != NO_LABEL
            label = torch.where(has, t[part], 0)
            h = s["hidden"][part].double()
            l = torch.matmul(h, w.mT)
            z = torch.logsumexp(l, 1)
            lse[part] = torch.where(has, z, 0.0)
            loss[part] = torch.where(has, z - l.gather(1, label[:, None])[:, 0], 0.0)
            if case["train"]:
                p = torch.softmax(l, 1).scatter_add(1, label[:, None], torch.full((len(label), 1), -1.0, dtype=torch.float64, device="cuda"))
                p *= torch.where(has, s["dloss"][part].double(), 0.0)[:, None]
                dh[part] = torch.matmul(p, w)
                dw += torch.matmul(p.mT, h)
        return (loss, lse, dh, dw) if case["train"] else (loss, lse)
    if case["op"] == "embed":
        ids, scale = s["ids"], s["scale"]
        if not case["grad"]:
            out = s["table"].double().index_select(0, ids) * scale
            out[ids == PAD] = 0.0
            return out
        total = s["dtable"].double() if case["accumulate"] else torch.zeros(case["V"], case["D"], dtype=torch.float64, device="cuda")
        keep = ids != PAD
        return total.index_put_((ids[keep],), s["dout"][keep].double() * scale, accumulate=True)
    x, dy = s["x"].double(), s["dy"].double()

    def both(v):
        u = math.sqrt(2.0 / math.pi) * (v + 0.044715 * v ** 3)
        th = torch.tanh(u)
        return 0.5 * v * (1.0 + th), 0.5 * (1.0 + th) + 0.5 * v * (1.0 - th * th) * math.sqrt(2.0 / math.pi) * (1.0 + 3 * 0.044715 * v ** 2)

    back = torch.empty_like(x)
    for lo in range(0, case["D"], 128):
        step = x[:, lo:lo + 128].abs().amax(1, keepdim=True) / 127.0
        back[:, lo:lo + 128] = torch.where(step > 0, torch.round(x[:, lo:lo + 128] / step) * step, 0.0)
    y_again, slope = both(back)
    return both(x)[0], dy * slope, y_again
