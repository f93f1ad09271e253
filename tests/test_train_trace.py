"""Calls of the training operators in a row under a kernel trace: every traced session gets to its end, and what the operators
return is what they return without a trace."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def api():
    from paper_2306_10598_b200 import build
    build.build_library()
    from paper_2306_10598_b200 import api
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return api


def passes(api, sets, count):
    for i in range(count):
        hidden, weight, targets, dloss, ids, x = sets[i % len(sets)]
        loss, lse = api.vocab_loss(hidden, weight, targets)
        dh, dw = api.vocab_loss_backward(hidden, weight, targets, lse, dloss)
        rows = api.embed_backward(dh, ids, weight.shape[0])
        y = api.gelu_save8(x)[0]
    torch.cuda.synchronize()
    return loss, lse, dh, dw, rows, y


@pytest.mark.parametrize("sessions", [((100, 8192), (8, 8192), (100, 8192)), ((8, 45976), (100, 45976), (300, 8000), (100, 45976))])
def test_traced_sessions_end(api, sessions):
    from torch.profiler import ProfilerActivity, profile

    for tokens, vocab in sessions:
        g = torch.Generator(device="cuda").manual_seed(tokens)
        sets = []
        for _ in range(3):
            hidden = torch.randn(tokens, 512, generator=g, device="cuda").bfloat16()
            weight = (torch.randn(vocab, 512, generator=g, device="cuda") / 512**0.5).bfloat16()
            targets = torch.randint(0, vocab, (tokens,), generator=g, device="cuda")
            sets.append((hidden, weight, targets, torch.full((tokens,), 1.0 / tokens, device="cuda"), targets, hidden))
        want = passes(api, sets, 6)
        with profile(activities=[ProfilerActivity.CUDA]) as trace:
            got = passes(api, sets, 12)
        assert sum(e.count for e in trace.key_averages() if "dct::" in e.key) >= 12 * 8
        for a, b in zip(want, got):
            assert torch.equal(a, b)
        assert api.dc_train_status() == 0
