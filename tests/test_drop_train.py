"""The training operators together: Algorithm 1's loop on the GPU, and the differentiable functions."""
import math

import pytest
import torch

import train_plain as plain

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def mods():
    from paper_2306_10598_b200 import build
    build.build_library()
    from paper_2306_10598_b200 import api, autograd, drop_train
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return api, autograd, drop_train


def test_micro_batches_accumulate_like_the_formula(mods):
    """Three micro-batches' gradients summed in fp32 against the whole chain in 64 bits."""
    _, _, dt = mods
    V, D = 301, 128
    g = torch.Generator(device="cuda").manual_seed(3)
    table, head = ((torch.randn(V, D, generator=g, device="cuda") / math.sqrt(D)).to(BF16) for _ in range(2))
    text = dt.Text(V, 5, "cuda")
    got = [torch.zeros(V, D, device="cuda") for _ in range(2)]
    want = [torch.zeros(V, D, dtype=torch.float64, device="cuda") for _ in range(2)]
    size = [torch.zeros_like(w) for w in want]
    for _ in range(3):
        ids, targets = text.batch(3, 40)
        dt.micro_batch(table, head, ids, targets, *got)
        t, i = targets.reshape(-1), ids.reshape(-1)
        s = math.sqrt(D)
        x = (plain.embed(table, i, s, 0)).to(BF16)
        q, sc = plain.save8(x)
        v = plain.load8(q, sc).double().cuda()
        y = plain.gelu(x.double()).to(BF16)
        dh, dw, _, _ = plain.vocab_backward(y, head, t, -100, 1.0, torch.ones(len(t), device="cuda"))
        dx = dh * plain.gelu_slope(v)
        gt, at, _ = plain.embed_backward(dx, i, V, s, 0)
        want[0] += gt
        want[1] += dw
        size[0] += at
        size[1] += dw.abs()
    # y, dy and dx are rounded to 16 bits on the way, each by up to 2^-8 of itself (y once more where it falls on the other
    # side of a rounding boundary), and g by 2^-8 of its largest element's size: a few such roundings over the whole sum
    for a, b, z in zip(got, want, size):
        assert float((a.double() - b).norm()) <= 4 * 2.0 ** -8 * float(z.norm())
        assert float((a.double() - b).norm()) <= 0.03 * float(b.norm())


def test_training_with_dropped_micro_batches_learns(mods):
    _, _, dt = mods
    log = dt.train(steps=30, workers=6, vocab=257, width=64, seed=2)
    assert all(0 < r["micro_batches"] <= r["planned"] for r in log)
    assert sum(r["micro_batches"] for r in log) < sum(r["planned"] for r in log)          # some were dropped
    assert all(r["step_time"] <= r["without_drop"] for r in log)
    assert log[0]["loss"] > 0.8 * math.log(256)
    assert log[-1]["loss"] < 0.5 * log[0]["loss"]


def test_run_until_is_the_simulators_count(mods):
    """What the loop runs is what the sweep counts as completed."""
    api, _, dt = mods
    from paper_2306_10598_b200 import workloads as W
    w = W.c3_workload("lognormal_0.05", N=40, T=50, K=16, t_comm=0.5, seed=4)
    lat = W.fill_latencies(w, "cuda")
    taus = torch.from_numpy(W.make_taus(w)).cuda()
    r = api.sweep(lat, taus, 0.5)
    for k in (0, 5, 15):
        ran = torch.stack([dt.run_until(lat[t], float(taus[k])).sum() for t in range(50)])
        assert torch.equal(ran, r.out_done[:, k].long())


def test_differentiable_functions(mods):
    """Gradients through the functions are those of the calls, also for the gradient of a mean, one value seen many times."""
    api, ag, _ = mods
    g = torch.Generator(device="cuda").manual_seed(8)
    table = (torch.randn(50, 64, generator=g, device="cuda") / 8).to(BF16).requires_grad_()
    head = (torch.randn(90, 64, generator=g, device="cuda") / 8).to(BF16).requires_grad_()
    ids = torch.randint(0, 50, (4, 9), generator=g, device="cuda")
    t = torch.randint(0, 90, (4, 9), generator=g, device="cuda")
    t[0, :4] = -100
    x = ag.embed(table, ids, 3.0, 7)
    y = ag.gelu(x)
    loss = ag.vocab_loss(y, head, t)
    loss.mean().backward()
    ev = api.embed(table.detach(), ids, 3.0, 7)
    s = api.gelu_save8(ev)
    l, lse = api.vocab_loss(s.y, head.detach(), t)
    assert torch.equal(loss, l) and torch.equal(x, ev)
    dy, dw = api.vocab_loss_backward(s.y, head.detach(), t, lse, torch.full_like(l, 1.0 / 36))
    dx = api.gelu_save8_backward(dy, s.q, s.scales)
    assert torch.equal(head.grad, dw) and torch.equal(table.grad, api.embed_backward(dx, ids, 50, 3.0, 7))
    # sequences without their last place, as next-token training slices them
    x2 = ag.gelu(ag.embed(table, ids[:, :-1], 3.0, 7))
    shifted = ag.vocab_loss(ag.gelu(ag.embed(table, ids, 3.0, 7))[:, :-1], head, t[:, 1:])
    assert torch.equal(shifted, ag.vocab_loss(x2, head, t[:, 1:].contiguous()))
    shifted.sum().backward()
    # a head that is not trained costs no gradient of its own
    frozen = ag.vocab_loss(y.detach().requires_grad_(), head.detach(), t)
    frozen.sum().backward()


def test_graph_replay_gives_the_same_bits(mods):
    """The calls neither allocate nor synchronise: captured once, replayed on new inputs."""
    api, _, _ = mods
    g = torch.Generator(device="cuda").manual_seed(9)
    N, V, D = 260, 700, 96
    h = torch.randn(N, D, generator=g, device="cuda").to(BF16)
    w = (torch.randn(V, D, generator=g, device="cuda") / 10).to(BF16)
    t = torch.randint(0, V, (N,), generator=g, device="cuda")
    dloss = torch.full((N,), 1.0 / N, device="cuda")
    loss, lse, dh, dw = torch.empty(N, device="cuda"), torch.empty(N, device="cuda"), torch.empty_like(h), torch.empty(V, D, device="cuda")
    dt = torch.empty(V, D, device="cuda")
    ws = torch.empty(max(api.dc_vocab_loss_workspace_bytes(N, w, b) for b in (False, True)), dtype=torch.uint8, device="cuda")
    we = torch.empty(api.dc_embed_backward_workspace_bytes(N, V, D), dtype=torch.uint8, device="cuda")

    def calls():
        api.dc_vocab_loss(h, w, t, loss, lse, ws)
        api.dc_vocab_loss_backward(h, w, t, lse, dloss, dh, dw, ws)
        api.dc_embed_backward(dh, t, dt, we)
    calls()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    h.copy_(torch.randn(N, D, generator=g, device="cuda"))
    t.copy_(torch.randint(0, V, (N,), generator=g, device="cuda"))
    t[5:40] = -100
    graph.replay()
    torch.cuda.synchronize()
    got = [x.clone() for x in (loss, lse, dh, dw, dt)]
    for x in (loss, lse, dh, dw, dt):
        x.fill_(7.0)
    calls()
    assert all(torch.equal(a, b) for a, b in zip(got, (loss, lse, dh, dw, dt)))
