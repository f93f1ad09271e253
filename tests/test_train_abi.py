"""include/dropcompute_train.h: every function exported and bound, and argument errors as status codes before anything is
enqueued (no GPU needed)."""
import ctypes
import os

import pytest

from test_library_abi import ROOT, declared_functions, lib  # noqa: F401

HEADER = os.path.join(ROOT, "include", "dropcompute_train.h")
A = 0x10000   # a made-up aligned address: validation fails before anything is dereferenced
NULL, SHAPE, ALIGN, RANGE, CUDA, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 6, 7, 9
F = ctypes.c_float(1.0)


def test_train_functions_are_exported(lib):  # noqa: F811
    from paper_2306_10598_b200 import api
    names = declared_functions(HEADER)
    assert sorted(api.TRAIN_EXPORTS) == names
    assert not set(names) & (set(api.EXPORTS) | set(api.DEV_EXPORTS))
    for n in names:
        assert hasattr(lib, n), f"{n} is declared in dropcompute_train.h but not exported"


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), SHAPE), (dict(V=0), SHAPE), (dict(D=0), SHAPE), (dict(N=1 << 31), RANGE), (dict(V=1 << 31), RANGE), (dict(D=1 << 31), RANGE),
    (dict(dtype=3), UNSUPPORTED), (dict(dtype=-1), UNSUPPORTED), (dict(table=None), NULL), (dict(ids=None), NULL), (dict(out=None), NULL),
    (dict(ts=7), SHAPE), (dict(os=7), SHAPE), (dict(table=A + 1), ALIGN), (dict(ids=A + 4), ALIGN), (dict(out=A + 1), ALIGN), (dict(N=0, table=None), 0)])
def test_embed_refusals(lib, change, status):  # noqa: F811
    a = dict(table=A, ts=8, dtype=0, ids=A, N=4, V=10, D=8, out=A, os=8) | change
    assert lib.dc_embed(a["table"], a["ts"], a["dtype"], a["ids"], a["N"], a["V"], a["D"], F, -1, a["out"], a["os"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), SHAPE), (dict(V=0), SHAPE), (dict(V=4194305), RANGE), (dict(N=1 << 31), RANGE), (dict(dtype=3), UNSUPPORTED), (dict(odt=1), UNSUPPORTED),
    (dict(dout=None), NULL), (dict(ids=None), NULL), (dict(dt=None), NULL), (dict(ds=7), SHAPE), (dict(dts=7), SHAPE), (dict(dout=A + 1), ALIGN),
    (dict(ids=A + 4), ALIGN), (dict(dt=A + 2), ALIGN), (dict(ws=None), WORKSPACE), (dict(ws=A + 16), WORKSPACE), (dict(wb=100), WORKSPACE),
    (dict(N=0, dout=None, ids=None, ws=None, acc=1), 0)])
def test_embed_backward_refusals(lib, change, status):  # noqa: F811
    a = dict(dout=A, ds=8, dtype=0, ids=A, N=4, V=10, D=8, dt=A, dts=8, odt=2, acc=1, ws=A, wb=1 << 20) | change
    assert lib.dc_embed_backward(a["dout"], a["ds"], a["dtype"], a["ids"], a["N"], a["V"], a["D"], F, -1, a["dt"], a["dts"], a["odt"], a["acc"],
                                 a["ws"], a["wb"], None) == status


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), SHAPE), (dict(D=0), SHAPE), (dict(N=1 << 31), RANGE), (dict(dtype=5), UNSUPPORTED), (dict(x=None), NULL), (dict(y=None), NULL),
    (dict(q=None), NULL), (dict(s=None), NULL), (dict(xs=3), SHAPE), (dict(ys=3), SHAPE), (dict(x=A + 1), ALIGN), (dict(s=A + 2), ALIGN), (dict(N=0, x=None), 0)])
def test_gelu_refusals(lib, change, status):  # noqa: F811
    a = dict(x=A, xs=8, dtype=0, N=4, D=8, y=A, ys=8, q=A, s=A) | change
    assert lib.dc_gelu_save8(a["x"], a["xs"], a["dtype"], a["N"], a["D"], a["y"], a["ys"], a["q"], a["s"], None) == status
    assert lib.dc_gelu_save8_backward(a["x"], a["xs"], a["dtype"], a["q"], a["s"], a["N"], a["D"], a["y"], a["ys"], None, 0, None) == status


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), SHAPE), (dict(V=0), SHAPE), (dict(D=0), SHAPE), (dict(V=1 << 31), RANGE), (dict(dtype=2), UNSUPPORTED), (dict(h=None), NULL),
    (dict(w=None), NULL), (dict(t=None), NULL), (dict(loss=None), NULL), (dict(lse=None), NULL), (dict(hs=7), SHAPE), (dict(ws=7), SHAPE),
    (dict(h=A + 1), ALIGN), (dict(w=A + 1), ALIGN), (dict(t=A + 4), ALIGN), (dict(loss=A + 2), ALIGN), (dict(work=None), WORKSPACE),
    (dict(work=A + 16), WORKSPACE), (dict(wb=1000), WORKSPACE)])
def test_vocab_loss_refusals(lib, change, status):  # noqa: F811
    a = dict(h=A, hs=8, w=A, ws=8, dtype=0, t=A, N=4, V=10, D=8, loss=A, lse=A, work=A, wb=1 << 40) | change
    assert lib.dc_vocab_loss(a["h"], a["hs"], a["w"], a["ws"], a["dtype"], a["t"], a["N"], a["V"], a["D"], -100, F, a["loss"], a["lse"],
                             a["work"], a["wb"], None) == status
    assert lib.dc_vocab_loss_backward(a["h"], a["hs"], a["w"], a["ws"], a["dtype"], a["t"], a["N"], a["V"], a["D"], -100, F, a["lse"], a["loss"],
                                      A, 8, A, 8, 2, 0, a["work"], a["wb"], None) == status


def test_vocab_loss_backward_refusals(lib):  # noqa: F811
    def call(dh=A, dhs=8, dw=A, dws=8, dwt=0, N=4):
        return lib.dc_vocab_loss_backward(A, 8, A, 8, 0, A, N, 10, 8, -100, F, A, A, dh, dhs, dw, dws, dwt, 1, A, 100, None)
    assert call(dh=None, dw=None) == NULL and call(dwt=1) == UNSUPPORTED and call(dhs=7) == SHAPE and call(dws=7) == SHAPE
    assert call(dh=A + 1) == ALIGN and call(dw=A + 2, dwt=2) == ALIGN and call() == WORKSPACE and call(N=0) == 0


def test_workspace_bytes(lib):  # noqa: F811
    assert lib.dc_embed_backward_workspace_bytes(-1, 4, 4) == 0 and lib.dc_embed_backward_workspace_bytes(4, 1 << 23, 4) == 0
    small, large = (lib.dc_embed_backward_workspace_bytes(n, 1000, 64) for n in (10, 10000))
    assert 0 < small < large < 10000 * 64 * 4                       # less than the gradient that is summed
    assert lib.dc_vocab_loss_workspace_bytes(4, 0, 4, A, 4, 0) == 0
    assert lib.dc_vocab_loss_workspace_bytes(0, 10, 4, A, 4, 0) > 0 and lib.dc_vocab_loss_workspace_bytes(0, 10, 4, A, 4, 1) > 0
    aligned, copied = (lib.dc_vocab_loss_workspace_bytes(100, 5000, 64, A + o, 64, 0) for o in (0, 2))
    assert copied - aligned >= 5000 * 64 * 2                        # the copy of a weight whose rows are off 16 bytes
    # the logits of 65536 x 262144 would be 32 GiB in 16 bits: neither direction needs a tenth of that
    assert lib.dc_vocab_loss_workspace_bytes(65536, 262144, 1024, A, 1024, 0) < (3 << 30)
    assert lib.dc_vocab_loss_workspace_bytes(65536, 262144, 1024, A, 1024, 1) < (3 << 30)
