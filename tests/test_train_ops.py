"""The training operators (include/dropcompute_train.h) on the GPU against their formulas in 64 bits."""
import math

import pytest
import torch

import train_plain as plain

pytestmark = pytest.mark.gpu

BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def api():
    from paper_2306_10598_b200 import build
    build.build_library()
    from paper_2306_10598_b200 import api as _api
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return _api


@pytest.fixture(autouse=True)
def no_wait_expired(api):
    yield
    api.dc_train_status()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


def spaced(t, gap, offset=0):
    """The same values in rows `gap` elements further apart, starting `offset` elements into their memory."""
    n, d = t.shape
    room = torch.full((n * (d + gap) + offset + 64,), 7.0, device=t.device).to(t.dtype)
    v = room[offset:offset + n * (d + gap)].view(n, d + gap)[:, :d]
    v.copy_(t)
    return v


def close(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound) & ~(got.double().isnan() & want.isnan())
    assert not bool(bad.any()), (what, int(bad.sum()), float((got.double() - want)[bad].abs().max()), bad.nonzero()[0].tolist())


# ---- embedding ----------------------------------------------------------------------------------------------------------

EMBED = [(1, 1, 1), (1, 5, 8), (3, 7, 3), (16, 100, 64), (33, 1000, 129), (257, 300, 1024), (1000, 50, 1032), (70, 9, 513), (40, 11, 4100), (0, 4, 8)]


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N,V,D", EMBED)
def test_embed(api, N, V, D, dtype):
    g = gen(N * 1000 + D)
    table = normal(g, V, D, dtype=dtype)
    ids = torch.randint(0, V, (N,), generator=g, device="cuda")
    if N >= 3:
        ids[1], ids[2] = V, -3                       # outside the table
    pad = int(ids[0]) if N else -1
    out = api.embed(table, ids, scale=1.7, pad_id=pad)
    want = plain.embed(table, ids, torch.tensor(1.7, dtype=F32).item(), pad)
    close(out, want, want.abs() * (plain.ROUND[dtype] + 2.0 ** -23) + plain.TINY[dtype], (N, V, D))
    again = api.embed(table, ids, scale=1.7)         # no padding token: a negative id matches nothing, not even -1
    assert torch.equal(again.isnan().all(-1), (ids < 0) | (ids >= V))
    if N:
        lowest = torch.full((1,), -(1 << 63), dtype=torch.int64, device="cuda")
        assert bool(api.embed(table, lowest).isnan().all())


def test_embed_strides_and_shapes(api):
    g = gen(5)
    for dtype in (BF16, F32):
        for D, gap, offset in ((64, 3, 1), (64, 8, 0), (65, 0, 1), (63, 1, 0)):
            table = normal(g, 40, D, dtype=dtype)
            ids = torch.randint(0, 40, (3, 7), generator=g, device="cuda")
            want = (table.float() * 0.5).to(dtype)[ids]
            out = spaced(torch.zeros(21, D, device="cuda", dtype=dtype), gap, offset)
            api.dc_embed(spaced(table, gap, offset), ids, out, scale=0.5)
            assert torch.equal(out.reshape(3, 7, D), want)
            if gap:                                   # what lies between the rows is left alone
                room = torch.as_strided(out, (21, D + gap), (D + gap, 1))[:, D:]
                assert bool((room == 7.0).all())


BACK = [(1, 1, 1), (5, 3, 8), (31, 40, 64), (32, 1, 72), (33, 2, 129), (64, 5, 40), (100, 4, 1024), (1000, 10, 96), (5000, 3, 40), (3000, 5003, 136),
        (20000, 40000, 8), (9000, 1, 16), (2049, 600000, 8)]


@pytest.mark.parametrize("dtype,out", [(BF16, F32), (BF16, BF16), (F16, F32), (F16, F16), (F32, F32)])
@pytest.mark.parametrize("N,V,D", BACK)
def test_embed_backward(api, N, V, D, dtype, out):
    g = gen(N + D)
    dout = normal(g, N, D, dtype=dtype)
    u = torch.rand(N, generator=g, device="cuda", dtype=torch.float64)
    ids = (torch.exp(u * math.log(V + 1)).long() - 1).clamp_(0, V - 1)     # a few tokens hold most places
    pad = -1
    if N >= 31:
        ids[3], ids[4], ids[7] = -1, V, 1 << 40
        pad = int(ids[0]) if V > 1 else -1
    scale = torch.tensor(0.3, dtype=F32).item()
    want, size, m = plain.embed_backward(dout, ids, V, scale, pad)
    got = api.embed_backward(dout, ids, V, scale=0.3, pad_id=pad, dtype=out)
    assert got.dtype == out
    bound = (m + 3) * 2.0 ** -24 * size + plain.ROUND[out] * want.abs() * 1.01 + plain.TINY[out]
    close(got, want, bound, (N, V, D))
    assert torch.equal(got, api.embed_backward(dout, ids, V, scale=0.3, pad_id=pad, dtype=out))          # the same bits again
    old = normal(g, V, D, dtype=out)
    acc = old.clone()
    assert api.embed_backward(dout, ids, V, scale=0.3, pad_id=pad, dtable=acc, accumulate=True) is acc
    both = old.double() + want
    close(acc, both, bound + plain.ROUND[out] * both.abs() * 1.01 + 2.0 ** -24 * (old.double().abs() + size), (N, V, D, "accumulated"))
    untouched = size.sum(1) == 0
    assert torch.equal(acc[untouched], old[untouched])


def test_embed_backward_edges(api):
    g = gen(9)
    table = torch.full((6, 10), NAN, device="cuda")
    api.embed_backward(torch.empty(0, 10, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda"), 6, dtable=table)
    assert bool((table == 0).all())                                         # no tokens: zeros
    ids = torch.full((50,), 2, device="cuda")
    d = normal(g, 50, 10)
    d[4] = NAN
    ids[4] = 3
    got = api.embed_backward(d, ids, 6, pad_id=3)                            # what padding holds is not used
    assert not bool(got.isnan().any()) and bool((got[[0, 1, 3, 4, 5]] == 0).all())
    got = api.embed_backward(d, torch.full((50,), 3, device="cuda"), 6, pad_id=3)   # nothing but padding
    assert bool((got == 0).all())
    # rows apart from each other on both sides
    for gap, offset in ((3, 1), (8, 0)):
        d = normal(g, 300, 64, dtype=BF16)
        ids = torch.randint(0, 20, (300,), generator=g, device="cuda")
        out = spaced(torch.zeros(20, 64, device="cuda"), gap, offset)
        api.embed_backward(spaced(d, gap, offset), ids, 20, dtable=out)
        assert torch.equal(out, api.embed_backward(d, ids, 20, dtype=F32))
        assert bool((torch.as_strided(out, (20, 64 + gap), (64 + gap, 1))[:, 64:] == 7.0).all())


def test_embed_gradient_against_differences(api):
    g = gen(11)
    V, D, N = 13, 24, 60
    table, ids, dout = normal(g, V, D), torch.randint(0, V, (N,), generator=g, device="cuda"), normal(g, N, D)
    grad = api.embed_backward(dout, ids, V, scale=2.5, pad_id=4)
    along = normal(g, V, D)
    f = lambda t: (plain.embed(t, ids, 2.5, 4) * dout.double()).sum()       # noqa: E731
    slope = (f(table.double() + along.double()) - f(table.double() - along.double())) / 2      # linear: any step will do
    terms = (plain.embed_backward(dout, ids, V, 2.5, 4)[1] * along.double().abs()).sum()
    assert abs(float(slope - (grad.double() * along.double()).sum())) <= 2.0 ** -24 * (N + 3) * float(terms)


# ---- gelu in 8 bits ------------------------------------------------------------------------------------------------------

GELU = [(1, 1), (1, 128), (3, 129), (5, 127), (2, 8), (67, 1001), (130, 264), (33, 1024), (700, 96), (0, 16)]


def gelu_bounds(v, dtype):
    """fp32 evaluation of the gate: exp(z) with a relative error of |z| 2^-23 + 2^-21, |z| = 2u; where the gate is far from 0 and 1
    that carries over, elsewhere it shrinks; plus the rounding of the result.  z is bounded by what exp turns into 0 or inf."""
    z = (2 * plain.A * (v + plain.B * v ** 3)).abs().clamp(max=90.0)
    rel = z * 2.0 ** -22 + 2.0 ** -20
    y, s = plain.gelu(v), plain.gelu_slope(v)
    gate_err = rel * 0.25 + 2.0 ** -22
    by = v.abs() * gate_err.minimum(torch.ones_like(v)) + plain.ROUND[dtype] * 1.01 * y.abs() + plain.TINY[dtype]
    bs = gate_err * (1.0 + v.abs() * 1.6 * (1.0 + 0.2 * v * v)).clamp(max=60.0)
    return y, by, s, bs


@pytest.mark.parametrize("dtype", [BF16, F16, F32])
@pytest.mark.parametrize("N,D", GELU)
def test_gelu_save8(api, N, D, dtype):
    g = gen(N * 7 + D)
    x = normal(g, N, D, dtype=dtype, scale=2.0)
    if N >= 3:
        x[0, :] = 0.0                         # a row without anything
        x[1] *= 2e-38 if dtype != F16 else 6e-8
        x[2, 0] = 300.0
    y, q, scales = api.gelu_save8(x)
    want_q, want_s = plain.save8(x)
    assert torch.equal(q.cpu(), want_q) and torch.equal(scales.cpu(), want_s)
    want, bound, _, _ = gelu_bounds(x.double(), dtype)
    close(y, want, bound, (N, D))
    dy = normal(g, N, D, dtype=dtype)
    dx, y_again = api.gelu_save8_backward(dy, q, scales, want_y=True)
    v = plain.load8(q, scales)                # fp32, as the operator defines it
    y2, by2, slope, bs = gelu_bounds(v.double(), dtype)
    close(y_again, y2, by2, (N, D, "again"))
    wdx = dy.double() * slope
    close(dx, wdx, dy.double().abs() * bs + plain.ROUND[dtype] * 1.01 * wdx.abs() + plain.TINY[dtype], (N, D, "dx"))
    assert torch.equal(dx, api.gelu_save8_backward(dy, q, scales))
    # what is read back is within half a step of x
    if D and N:
        step = scales.double().repeat_interleave(128, 1)[:, :D]
        tiny = x.double().abs() * (step == 0)
        close(v.double(), x.double(), step * 0.5001 + tiny, (N, D, "step"))


def test_gelu_save8_strides_and_non_finite(api):
    g = gen(3)
    for dtype in (BF16, F32):
        for D, gap, offset in ((256, 3, 1), (256, 8, 0), (200, 8, 8), (100, 0, 1)):
            x, dy = normal(g, 9, D, dtype=dtype), normal(g, 9, D, dtype=dtype)
            y, q, s = api.gelu_save8(x)
            y2, q2, s2 = spaced(torch.zeros_like(x), gap, offset), torch.zeros_like(q), torch.zeros_like(s)
            api.dc_gelu_save8(spaced(x, gap, offset), y2, q2, s2)
            assert torch.equal(y, y2) and torch.equal(q, q2) and torch.equal(s, s2)
            dx = spaced(torch.zeros_like(x), gap, offset)
            api.dc_gelu_save8_backward(spaced(dy, gap, offset), q, s, dx)
            assert torch.equal(dx, api.gelu_save8_backward(dy, q, s))
    for bad in (NAN, INF, -INF):
        x = normal(g, 4, 300, dtype=BF16)
        x[1, 130] = bad
        y, q, s = api.gelu_save8(x)
        assert bool(s[1, 1].isnan()) and int(s.isnan().sum()) == 1 and bool((q[1, 128:256] == 0).all())
        dx, again = api.gelu_save8_backward(torch.ones_like(x), q, s, want_y=True)
        hit = torch.zeros(4, 300, dtype=torch.bool, device="cuda")
        hit[1, 128:256] = True
        assert torch.equal(dx.isnan(), hit) and torch.equal(again.isnan(), hit)
    big = torch.tensor([[3e38, -3e38, 1.0, -1e20, 1e20]], device="cuda", dtype=BF16)
    y, q, s = api.gelu_save8(big)
    assert y.float().tolist()[0][0] == float(big[0, 0]) and float(y[0, 1]) == 0.0
    dx = api.gelu_save8_backward(torch.ones_like(big), q, s)
    assert dx.float().tolist()[0] == [1.0, 0.0, 0.5, 0.5, 0.5]              # 1, -1e20 and 1e20 read back as 0


def test_gelu_slope_against_differences(api):
    g = gen(4)
    x, dy = normal(g, 20, 200, scale=1.5), normal(g, 20, 200)
    _, q, s = api.gelu_save8(x)
    dx = api.gelu_save8_backward(dy, q, s)
    v = plain.load8(q, s).double()
    h = 1e-5
    slope = (plain.gelu(v + h) - plain.gelu(v - h)) / (2 * h)               # its own error: h^2/6 |f'''| + 2^-52 / h < 1e-9
    _, _, _, bs = gelu_bounds(v, F32)
    close(dx, dy.double() * slope, dy.double().abs() * (bs + 1e-9 + 2.0 ** -24 * 1.2), "differences")


# ---- vocabulary loss ------------------------------------------------------------------------------------------------------

def make_loss(N, V, D, dtype, seed, keep=1.0, wscale=None, ignore=-100):
    g = gen(seed)
    w = normal(g, V, D, scale=wscale or 1.0 / math.sqrt(D))
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    h = normal(g, N, D) + torch.rand(N, 1, generator=g, device="cuda") * 6 * w[t]
    if keep < 1.0:
        t[torch.rand(N, generator=g, device="cuda") >= keep] = ignore
    dloss = (torch.rand(N, generator=g, device="cuda") + 0.5) / max(1, N)
    return h.to(dtype), w.to(dtype), t, dloss


def check_forward(api, h, w, t, ignore=-100, c=1.0):
    loss, lse = api.vocab_loss(h, w, t, ignore_index=ignore, logit_scale=c)
    wl, wz, rows, l = plain.vocab_loss(h, w, t, ignore, torch.tensor(c, dtype=F32).item())
    e = plain.vocab_logit_error(h, w, rows, c)
    # lse: the logits' error, and exp and log in fp32 with arguments up to the logits' range
    span = (l.amax(1) - l.amin(1)).clamp(max=90.0) if len(rows) else e
    ez = e + span * 2.0 ** -22 + 2.0 ** -18 + wz[rows].abs() * 2.0 ** -22
    bound = torch.zeros_like(wl)
    bound[rows] = ez
    close(lse, wz, bound, "lse")
    bound[rows] = ez + e + wl[rows].abs() * 2.0 ** -22
    close(loss, wl, bound, "loss")
    return loss, lse, e, span


def check_backward(api, h, w, t, dloss, lse, e, span, ignore=-100, c=1.0, dw_dtype=None):
    c32 = torch.tensor(c, dtype=F32).item()
    dt = h.dtype
    dh, dw = api.vocab_loss_backward(h, w, t, lse, dloss, ignore_index=ignore, logit_scale=c,
                                     dweight=None if dw_dtype is None else torch.full(w.shape, NAN, device="cuda", dtype=dw_dtype))
    wdh, wdw, g, rows = plain.vocab_backward(h, w, t, ignore, c32, dloss)
    V = w.shape[0]
    # g = (p - [label]) d: p is off by its exponent's error (logit, lse, exp), g by its rounding to 16 bits and, in fp16, by what falls
    # below the smallest subnormal of the scaled type
    p = g.clone()
    at = torch.arange(len(rows), device="cuda")
    d = (dloss[rows].double() * c32)[:, None]
    p[at, t[rows]] += d[:, 0]
    amax = float(d.abs().max()) if len(rows) else 0.0
    eg = p.abs() * (3 * e + span * 2.0 ** -21 + 2.0 ** -17)[:, None] + g.abs() * (plain.ROUND[dt] * 1.01 + 2.0 ** -21) + \
        d.abs() * 2.0 ** -23 * (p.abs() > 0) * (g.abs() < p.abs()) + (amax * 2.0 ** -38 if dt == F16 else 2.0 ** -133)
    hd, wd = h[rows].double(), w.double()
    bh = torch.zeros_like(wdh)
    bh[rows] = eg @ wd.abs() + (V + 64) * 2.0 ** -22 * (g.abs() @ wd.abs())
    close(dh, wdh, bh + plain.ROUND[dt] * 1.01 * wdh.abs() + plain.TINY[dt], "dhidden")
    out = dw.dtype
    # the rows' weights are brought into h before the product, which rounds it to 16 bits once more
    bw = eg.t() @ hd.abs() + ((len(rows) + 64) * 2.0 ** -22 + plain.ROUND[dt] * 1.01) * (g.abs().t() @ hd.abs())
    bw = bw + (amax * 2.0 ** -25 * (g / d).abs().sum(0)[:, None] if dt == F16 else 0.0)
    close(dw, wdw, bw + plain.ROUND[out] * 1.01 * wdw.abs() + plain.TINY[out], "dweight")
    return dh, dw, wdw, bw


LOSS = [(1, 1, 1), (1, 2, 8), (2, 7, 64), (31, 255, 63), (32, 256, 64), (33, 257, 65), (64, 1000, 128), (65, 5003, 129), (127, 300, 200), (128, 512, 72),
        (129, 513, 264), (255, 130, 1024), (256, 2048, 320), (257, 4097, 136), (600, 777, 96), (1025, 1500, 520), (9, 32000, 256), (300, 9, 1032),
        # few tokens: one pass over the weight, up to 16 of them and as long as their rows fit
        (1, 5000, 1024), (3, 70001, 72), (5, 1000, 1032), (8, 17, 40), (16, 4097, 200), (17, 300, 520), (32, 5003, 1024), (15, 5003, 1024), (16, 40, 3080), (7, 100, 6152), (33, 1000, 1024)]


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("N,V,D", LOSS)
def test_vocab_loss(api, N, V, D, dtype):
    h, w, t, dloss = make_loss(N, V, D, dtype, N + V + D)
    _, lse, e, span = check_forward(api, h, w, t)
    check_backward(api, h, w, t, dloss, lse, e, span)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("keep,ignore", [(0.15, -100), (0.5, 0), (0.9, 1 << 40), (0.0, -1)])
def test_vocab_loss_rows_without_a_label(api, keep, ignore, dtype):
    N, V, D = 700, 601, 136
    h, w, t, dloss = make_loss(N, V, D, dtype, 17, keep=keep, ignore=ignore)
    free = t == ignore
    h[free] = torch.tensor([NAN, INF, -INF, 1.0], device="cuda", dtype=dtype).repeat(D // 4)     # what they hold is not used
    dloss[free] = NAN
    _, lse, e, span = check_forward(api, h, w, t, ignore)
    lse = torch.where(free, torch.full_like(lse, NAN), lse)
    h0, d0 = torch.where(free[:, None], torch.zeros_like(h), h), torch.where(free, torch.zeros_like(dloss), dloss)
    dh, dw = api.vocab_loss_backward(h, w, t, lse, dloss, ignore_index=ignore)
    dh0, dw0 = api.vocab_loss_backward(h0, w, t, lse.nan_to_num(), d0, ignore_index=ignore)
    assert torch.equal(dh, dh0) and torch.equal(dw, dw0) and bool((dh[free] == 0).all())
    check_backward(api, h0, w, t, d0, lse, e, span, ignore)
    if keep == 0.0:
        assert bool((dw == 0).all())


@pytest.mark.parametrize("dtype", [BF16, F16])
def test_vocab_loss_few_tokens_without_a_label(api, dtype):
    for N in (1, 6, 20, 32):
        h, w, t, _ = make_loss(N, 900, 264, dtype, N)
        t[::3] = -100
        h[::3] = NAN
        if N > 4:
            t[1], t[4] = 900, -7
        loss, lse, _, _ = check_forward(api, h, w, t)
        assert bool((loss[::3] == 0).all()) and bool((lse[::3] == 0).all())
        hs, ws = spaced(h, 8), spaced(w, 8)
        again = api.vocab_loss(hs, ws, t)
        assert torch.equal(again.loss.nan_to_num(5.0), loss.nan_to_num(5.0)) and torch.equal(again.lse.nan_to_num(5.0), lse.nan_to_num(5.0))
        t[:] = -100
        assert bool((api.vocab_loss(h, w, t).loss == 0).all())


def test_vocab_loss_targets_outside(api):
    h, w, t, dloss = make_loss(50, 90, 64, BF16, 1)
    t[3], t[7], t[49] = 90, -1, -(1 << 40)
    loss, lse, e, span = check_forward(api, h, w, t)
    assert loss.isnan().nonzero()[:, 0].tolist() == [3, 7, 49]
    dh, *_ = check_backward(api, h, w, t, dloss, lse, e, span)
    assert bool((dh[[3, 7, 49]] == 0).all())
    h[5, 2] = NAN                                   # a labelled row that holds a NaN spoils itself alone
    loss, _ = api.vocab_loss(h, w, t)
    assert loss.isnan().nonzero()[:, 0].tolist() == [3, 5, 7, 49]


@pytest.mark.parametrize("c,wscale", [(0.125, 1.0), (1.0, 3.0), (-1.5, 0.1), (30.0, 0.2)])
def test_vocab_loss_scales(api, c, wscale):
    """Flat and very peaked softmax, and a logit scale."""
    for dtype in (BF16, F16):
        h, w, t, dloss = make_loss(200, 1111, 72, dtype, 23, wscale=wscale)
        _, lse, e, span = check_forward(api, h, w, t, c=c)
        check_backward(api, h, w, t, dloss, lse, e, span, c=c)


def test_vocab_loss_lowest_and_infinite_logits(api):
    """A vocabulary entry at the type's lowest value, and one at -inf, drop out of the sum; a row of +inf is not finite."""
    h = torch.ones(40, 64, device="cuda", dtype=BF16)
    w = normal(gen(2), 700, 64, dtype=BF16, scale=0.1)
    w[300] = torch.finfo(BF16).min
    w[1] = 0
    w[1, 0] = -INF
    w[512:700] = 0
    w[512:700, 0] = -INF                            # a tile with nothing finite in it
    t = torch.full((40,), 5, device="cuda")
    loss, lse = api.vocab_loss(h, w, t)
    keep = [v for v in range(512) if v not in (1, 300)]
    wl, wz, *_ = plain.vocab_loss(h, w[keep], torch.full((40,), keep.index(5), device="cuda"), -100, 1.0)
    close(loss, wl, torch.full_like(wl, 1e-4), "loss")          # logits of about 1, 64 terms: 64 2^-22 + exp, log
    close(lse, wz, torch.full_like(wz, 1e-4), "lse")
    h[7, 0] = INF
    w[9] = 1.0
    w[1], w[512:700] = 0, 0
    assert not bool(api.vocab_loss(h, w, t).loss[7].isfinite())


@pytest.mark.parametrize("N", [4, 40])
def test_vocab_loss_label_at_minus_infinity(api, N):
    """A label whose logit is -inf: its loss is +inf, lse and the other rows are as they would be."""
    h = normal(gen(3), N, 64, dtype=BF16)
    h[:, 0] = 1.0
    w = normal(gen(4), 300, 64, dtype=BF16, scale=0.1)
    w[7] = 0
    w[7, 0] = -INF
    h[:, 1:] = h[:, 1:].abs() + 0.01                # no zero meets the infinity
    w[7, 1:] = -0.5
    t = torch.full((N,), 5, device="cuda")
    t[2] = 7
    loss, lse = api.vocab_loss(h, w, t)
    assert float(loss[2]) == INF and bool(lse.isfinite().all()) and bool(loss[torch.arange(N, device="cuda") != 2].isfinite().all())
    keep = [v for v in range(300) if v != 7]
    _, wz, *_ = plain.vocab_loss(h, w[keep], torch.full((N,), 5, device="cuda"), -100, 1.0)
    close(lse, wz, torch.full_like(wz, 1e-4), "lse")          # 64 terms of about 0.1: 64 2^-22, exp, log
    dh, dw = api.vocab_loss_backward(h, w, t, lse, torch.ones(N, device="cuda"), want_dhidden=True)
    assert bool(dw.isfinite().all())


def test_vocab_loss_strides_types_and_accumulation(api):
    for dtype in (BF16, F16):
        for D, gap, offset in ((64, 3, 1), (64, 8, 0), (129, 0, 0), (72, 1, 3)):
            h, w, t, dloss = make_loss(90, 333, D, dtype, D, keep=0.8)
            a = api.vocab_loss(h, w, t)
            hs, wsp = spaced(h, gap, offset), spaced(w, gap, offset)
            b = api.vocab_loss(hs, wsp, t)
            assert torch.equal(a.loss, b.loss) and torch.equal(a.lse, b.lse)
            dh, dw = api.vocab_loss_backward(h, w, t, a.lse, dloss)
            dh2, dw2 = spaced(torch.zeros_like(h), gap, offset), spaced(torch.zeros_like(w), gap, offset)
            ws = torch.empty(api.dc_vocab_loss_workspace_bytes(90, wsp, True), dtype=torch.uint8, device="cuda")
            api.dc_vocab_loss_backward(hs, wsp, t, a.lse, dloss, dh2, dw2, ws)
            assert torch.equal(dh, dh2) and torch.equal(dw, dw2)
            if gap:
                assert bool((torch.as_strided(dw2, (333, D + gap), (D + gap, 1))[:, D:] == 7.0).all())
                assert bool((torch.as_strided(dh2, (90, D + gap), (D + gap, 1))[:, D:] == 7.0).all())
            # each gradient alone, and in fp32 with what was there before
            assert torch.equal(api.vocab_loss_backward(h, w, t, a.lse, dloss, want_dweight=False)[0], dh)
            assert torch.equal(api.vocab_loss_backward(h, w, t, a.lse, dloss, want_dhidden=False)[1], dw)
            _, full = api.vocab_loss_backward(h, w, t, a.lse, dloss, dweight=torch.full(w.shape, NAN, device="cuda"))
            assert torch.equal(full.to(dtype), dw)
            old = normal(gen(1), *w.shape, scale=1e-2)
            acc = old.clone()
            api.vocab_loss_backward(h, w, t, a.lse, dloss, dweight=acc, accumulate=True)
            close(acc, old.double() + full.double(), (old.double().abs() + full.double().abs()) * 2.0 ** -23, "accumulated")
            acc16 = old.to(dtype)
            api.vocab_loss_backward(h, w, t, a.lse, dloss, dweight=acc16, accumulate=True)
            want = old.to(dtype).double() + full.double()
            close(acc16, want, want.abs() * plain.ROUND[dtype] * 1.01 + (old.double().abs() + full.double().abs()) * 2.0 ** -22 + plain.TINY[dtype], "16 bits")


def test_vocab_loss_several_pieces(api):
    """More than one piece of the vocabulary, the last one short."""
    h, w, t, dloss = make_loss(8192, 37001, 64, BF16, 77, keep=0.97)
    _, lse, e, span = check_forward(api, h, w, t)
    dh, dw, _, _ = check_backward(api, h, w, t, dloss, lse, e, span)
    again = api.vocab_loss_backward(h, w, t, lse, dloss)
    assert torch.equal(dh, again[0]) and torch.equal(dw, again[1])          # the same bits again


def test_vocab_loss_nothing(api):
    w = normal(gen(1), 10, 16, dtype=BF16)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    h = torch.empty(0, 16, dtype=BF16, device="cuda")
    r = api.vocab_loss(h, w, none)
    assert r.loss.shape == (0,)
    dh, dw = api.vocab_loss_backward(h, w, none, r.lse, r.loss)
    assert dh.shape == (0, 16) and bool((dw == 0).all())
    keep = torch.ones_like(w)
    api.vocab_loss_backward(h, w, none, r.lse, r.loss, dweight=keep, accumulate=True)
    assert bool((keep == 1).all())


def test_vocab_loss_gradient_against_differences(api):
    """The kernel's gradients along random directions against central differences of the 64-bit loss."""
    N, V, D = 60, 400, 48
    h, w, t, dloss = make_loss(N, V, D, BF16, 31, keep=0.8)
    _, lse, e, span = check_forward(api, h, w, t)
    dh, dw, wdw, bw = check_backward(api, h, w, t, dloss, lse, e, span, dw_dtype=F32)
    g = gen(6)
    f = lambda a, b: (plain.vocab_loss(a, b, t, -100, 1.0)[0] * dloss.double()).sum()       # noqa: E731
    s = 1e-4
    ah, aw = normal(g, N, D).double(), normal(g, V, D).double()
    slope_h = (f(h.double() + s * ah, w) - f(h.double() - s * ah, w)) / (2 * s)
    slope_w = (f(h, w.double() + s * aw) - f(h, w.double() - s * aw)) / (2 * s)
    # the bounds of the elements, summed along the direction, plus the difference's own s^2 term (about 1e-8 times 60 logits' spread)
    assert abs(float(slope_w - (dw.double() * aw).sum())) <= float((bw * aw.abs()).sum()) + 1e-6
    rel = float((dh.double() * ah).abs().sum()) * 2.0 ** -7
    assert abs(float(slope_h - (dh.double() * ah).sum())) <= rel + 1e-6


# ---- streams, threads, together --------------------------------------------------------------------------------------------

def test_on_another_stream(api):
    h, w, t, dloss = make_loss(300, 2000, 128, BF16, 5)
    ids = t.clone()
    want = api.vocab_loss(h, w, t), api.embed(w, ids), api.embed_backward(h, ids, 2000), api.gelu_save8(h)
    grads = api.vocab_loss_backward(h, w, t, want[0].lse, dloss)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        for _ in range(3):
            got = api.vocab_loss(h, w, t), api.embed(w, ids), api.embed_backward(h, ids, 2000), api.gelu_save8(h)
            back = api.vocab_loss_backward(h, w, t, got[0].lse, dloss)
    s.synchronize()
    assert torch.equal(got[0].loss, want[0].loss) and torch.equal(got[1], want[1]) and torch.equal(got[2], want[2])
    assert torch.equal(got[3].q, want[3].q) and torch.equal(back[0], grads[0]) and torch.equal(back[1], grads[1])


def test_offsets_beyond_32_bits(api):
    """Matrices of more than 2^31 elements: the last rows are what they would be alone."""
    g = gen(40)
    D = 2048
    N = (1 << 31) // D + 300
    table = normal(g, 70, D, dtype=BF16)
    ids = torch.randint(0, 70, (N,), generator=g, device="cuda")
    out = api.embed(table, ids, scale=2.0)
    assert torch.equal(out[-300:], api.embed(table, ids[-300:], scale=2.0))
    y, q, s = api.gelu_save8(out)
    y1, q1, s1 = api.gelu_save8(out[-300:].clone())
    assert torch.equal(y[-300:], y1) and torch.equal(q[-300:], q1) and torch.equal(s[-300:], s1)
    dx = api.gelu_save8_backward(out, q, s)
    assert torch.equal(dx[-300:], api.gelu_save8_backward(out[-300:].clone(), q1, s1))
    del y, q, s, dx
    # rows of the last places alone: the same loss; labels elsewhere are missing, so the gradients are theirs too
    w = normal(g, 300, D, dtype=BF16, scale=0.02)
    t = torch.full((N,), -100, device="cuda")
    t[-300:] = torch.randint(0, 300, (300,), generator=g, device="cuda")
    dloss = torch.full((N,), 1.0 / 300, device="cuda")
    loss, lse = api.vocab_loss(out, w, t)
    alone = api.vocab_loss(out[-300:].clone(), w, t[-300:].clone())
    assert torch.equal(loss[-300:], alone.loss) and bool((loss[:-300] == 0).all())
    dh, dw = api.vocab_loss_backward(out, w, t, lse, dloss)
    dh1, dw1 = api.vocab_loss_backward(out[-300:].clone(), w, t[-300:].clone(), alone.lse, dloss[-300:].clone())
    assert torch.equal(dw, dw1) and bool((dh[:-300] == 0).all())
    rel = float((dh[-300:].float() - dh1.float()).norm() / dh1.float().norm())      # the vocabulary may be cut in other parts
    assert rel <= 2.0 ** -8
    del out, dh
    # a table of more than 2^31 elements
    V = (1 << 31) // 1024 + 50
    d = normal(g, 64, 1024)
    at = torch.randint(V - 40, V, (64,), generator=g, device="cuda")
    grad = api.embed_backward(d, at, V)
    assert torch.equal(grad[-40:], api.embed_backward(d, at - (V - 40), 40)) and bool((grad[:100] == 0).all()) and bool((grad[-60:-40] == 0).all())


def test_refusals(api):
    h, w, t, dloss = make_loss(8, 50, 64, BF16, 5)
    f = torch.zeros(8, device="cuda")
    with pytest.raises(TypeError):
        api.vocab_loss(h, w.half(), t)                        # two types
    with pytest.raises(TypeError):
        api.vocab_loss(h, w, t.int())
    with pytest.raises(TypeError):
        api.vocab_loss(h.cpu(), w, t)
    with pytest.raises(ValueError):
        api.vocab_loss(h, w[:, :32], t)
    with pytest.raises(ValueError):
        api.vocab_loss(h, w, t[:5])
    with pytest.raises(ValueError):
        api.vocab_loss(h, w.t().contiguous().t(), t)          # elements of a row apart
    with pytest.raises(ValueError):
        api.vocab_loss(h.view(2, 4, 64)[:, :3], w, t[:6])     # rows not evenly spaced
    with pytest.raises(api.DropComputeError) as x:
        api.vocab_loss(h.float(), w.float(), t)
    assert x.value.status == 7
    with pytest.raises(api.DropComputeError) as x:
        api.dc_vocab_loss(h, w, t, f, f.clone(), torch.empty(256, dtype=torch.uint8, device="cuda"))
    assert x.value.status == 9
    with pytest.raises(api.DropComputeError) as x:
        api.dc_vocab_loss_backward(h, w, t, f, dloss, None, None, torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    assert x.value.status == 1
    with pytest.raises(api.DropComputeError) as x:
        api.vocab_loss_backward(h, w, t, f, dloss, dweight=torch.zeros(50, 64, device="cuda", dtype=F16))
    assert x.value.status == 7
    with pytest.raises(ValueError):
        api.vocab_loss_backward(h, w, t, f, dloss, accumulate=True)
    with pytest.raises(TypeError):
        api.embed(w, t.int())
    with pytest.raises(ValueError):
        api.dc_embed(w, t, torch.empty(8, 32, device="cuda", dtype=BF16))
    with pytest.raises(ValueError):
        api.embed_backward(h, t[:3], 50)
    with pytest.raises(api.DropComputeError):
        api.embed_backward(h, t, 50, dtype=F16)
    with pytest.raises(ValueError):
        api.dc_gelu_save8(h, torch.empty_like(h), torch.empty(8, 32, device="cuda", dtype=torch.int8), torch.empty(8, 1, device="cuda"))
    with pytest.raises(TypeError):
        api.gelu_save8(h.double())
