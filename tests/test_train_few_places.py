"""The embedding's gradient where few places are summed without grouping, on both sides of the size where that ends."""
import pytest
import torch

import train_plain as plain

pytestmark = pytest.mark.gpu
BF16, F16, F32 = torch.bfloat16, torch.float16, torch.float32


@pytest.fixture(scope="module")
def api():
    from paper_2306_10598_b200 import build
    build.build_library()
    from paper_2306_10598_b200 import api
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    return api


def tokens(kind, N, V, g):
    if kind == "one":                                     # every place the same token
        return torch.full((N,), V - 1, device="cuda")
    if kind == "apart":                                   # no token twice, as far as there are as many
        return torch.randperm(max(N, V), generator=g, device="cuda")[:N] % V
    ids = torch.randint(0, V, (N,), generator=g, device="cuda")
    ids[torch.rand(N, generator=g, device="cuda") < 0.4] = V // 2
    return ids


SIZES = [(1, 1, 1), (2, 5, 33), (8, 300, 8), (9, 70, 257), (16, 3, 512), (17, 3, 513), (130, 40, 1000), (128, 2000, 136), (511, 90, 264),
         (512, 600, 69), (512, 7, 1024), (513, 7, 1024)]


@pytest.mark.parametrize("dtype,out", [(BF16, F32), (F16, F16), (BF16, BF16), (F32, F32)])
@pytest.mark.parametrize("kind", ["one", "apart", "often"])
@pytest.mark.parametrize("N,V,D", SIZES)
def test_sums_of_few_places(api, N, V, D, kind, dtype, out):
    g = torch.Generator(device="cuda").manual_seed(N * 7 + D)
    dout = torch.randn(N, D, generator=g, device="cuda").to(dtype)
    ids = tokens(kind, N, V, g)
    pad = -1
    if N >= 16 and kind != "one":
        pad = int(ids[5])
        dout[ids == pad] = float("nan")                   # what padding and ids outside the table hold is not used
        ids[2], ids[3], ids[11] = -3, V, 1 << 40
        dout[[2, 3, 11]] = float("inf")
    used = torch.where(torch.isfinite(dout), dout, torch.zeros_like(dout))
    scale = torch.tensor(-1.3, dtype=F32).item()
    want, size, m = plain.embed_backward(used, ids, V, scale, pad)
    got = api.embed_backward(dout, ids, V, scale=-1.3, pad_id=pad, dtype=out)
    # m - 1 additions, the multiplication, and the rounding of the result
    bound = (m + 3) * 2.0 ** -24 * size + plain.ROUND[out] * want.abs() * 1.01 + plain.TINY[out]
    assert bool(((got.double() - want).abs() <= bound).all())
    assert torch.equal(got, api.embed_backward(dout, ids, V, scale=-1.3, pad_id=pad, dtype=out))
    old = torch.randn(V, D, generator=g, device="cuda").to(out)
    acc = old.clone()
    api.embed_backward(dout, ids, V, scale=-1.3, pad_id=pad, dtable=acc, accumulate=True)
    both = old.double() + want
    assert bool(((acc.double() - both).abs() <= bound + plain.ROUND[out] * both.abs() * 1.01 + 2.0 ** -24 * (old.double().abs() + size)).all())
    untouched = size.sum(1) == 0
    assert torch.equal(acc[untouched], old[untouched]) and bool((got[untouched] == 0).all())


@pytest.mark.parametrize("V", [600000, 4194304])
def test_few_places_of_a_large_table(api, V):
    ids = torch.tensor([0, V - 1, 4095, 4096, V - 1, V // 2], device="cuda")
    dout = torch.arange(1.0, 7.0, device="cuda").reshape(6, 1)
    table = torch.full((V, 1), float("nan"), device="cuda")
    api.embed_backward(dout, ids, V, dtable=table)
    assert float(table[0]) == 1.0 and float(table[V - 1]) == 7.0 and float(table[4095]) == 3.0 and float(table[4096]) == 4.0 and float(table[V // 2]) == 6.0
    assert float(table.sum()) == 21.0 and int((table != 0).sum()) == 5


def test_few_places_with_rows_apart(api):
    g = torch.Generator(device="cuda").manual_seed(3)
    dout = torch.randn(200, 64, generator=g, device="cuda").bfloat16()
    ids = torch.randint(0, 9, (200,), generator=g, device="cuda")
    want = api.embed_backward(dout, ids, 9, dtype=F32)
    for gap, offset in ((3, 1), (8, 0), (8, 8)):
        room = torch.full((200 * (64 + gap) + offset,), 5.0, device="cuda", dtype=BF16)
        rows = torch.as_strided(room, (200, 64), (64 + gap, 1), offset)
        rows.copy_(dout)
        into = torch.full((9 * (64 + gap) + offset,), 7.0, device="cuda")
        out = torch.as_strided(into, (9, 64), (64 + gap, 1), offset)
        api.embed_backward(rows, ids, 9, dtable=out)
        assert torch.equal(out, want)
        assert int((into == 7.0).sum()) == into.numel() - out.numel()
