"""Host-side checks of the convolution's and the scan's entry points: sizes of their buffers, and bad
arguments turned down before anything is enqueued (no call reaches a kernel)."""
import ctypes
import os

import pytest
import torch

from paper_2011_13824_amd import blocks, lirpa

P = 0x10000  # stands for a device pointer: only its alignment is looked at
ODD = P + 1


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lirpa.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return lirpa.load()


CONV_BAD = [
    dict(dtype=3), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(n=0), dict(taps=0), dict(taps=9),
    dict(x=None), dict(x=ODD), dict(ldx=7), dict(w=None), dict(w=ODD), dict(bias=ODD), dict(act=2),
    dict(act=-1), dict(seq=P + 2), dict(slots=0), dict(state=ODD), dict(state_out=ODD),
    dict(y=None), dict(ldy=3), dict(ldy=1 << 22)]


@pytest.mark.parametrize("bad", CONV_BAD)
@pytest.mark.parametrize("call", ["lirpa_conv_forward", "lirpa_conv_step"])
def test_conv_refusals(L, bad, call):
    a = dict(dtype=lirpa.BF16, rows=4, n=8, taps=4, x=P, ldx=8, w=P, bias=P, act=1, seq=P, slots=3,
             state=P, state_out=P, y=P, ldy=8)
    a.update(bad)
    assert getattr(L, call)(*a.values(), None) == lirpa.LIRPA_EINVAL
    assert call in lirpa.lirpa_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=3), -1), (dict(rows=-1), -1), (dict(taps=9), -1), (dict(dy=None), -1),
    (dict(lddy=7), -1), (dict(x=None), -1), (dict(w=None), -1), (dict(act=7), -1),
    (dict(seq=ODD), -1), (dict(slots=0), -1), (dict(dx=None), -1), (dict(lddx=2), -1),
    (dict(dw=None), -1), (dict(dbias=ODD), -1), (dict(ws=None), -1), (dict(ws=P + 8), -1),
    (dict(ws_bytes=16), -2)])
def test_conv_backward_refusals(L, bad, code):
    a = dict(dtype=lirpa.F16, rows=4, n=8, taps=4, dy=P, lddy=8, x=P, ldx=8, w=P, bias=P, act=1,
             seq=P, slots=3, dx=P, lddx=8, dw=P, dbias=P, ws=P, ws_bytes=1 << 30)
    a.update(bad)
    assert L.lirpa_conv_backward(*a.values(), None) == code


def scan(**kw):
    a = dict(dtype=lirpa.BF16, rows=100, n=8, states=16, u=P, dt=P, z=P, B=P, C=P, ldu=8, lddt=8,
             ldz=8, ldB=16, ldC=16, A=P, D=P, bias=P, seq=P, slots=3)
    a.update(kw)
    return ctypes.byref(lirpa.lirpa_scan(*(a[k] for k, _ in lirpa.lirpa_scan._fields_)))


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(rows=-1), dict(n=0), dict(states=0), dict(states=65), dict(u=None),
    dict(u=ODD), dict(ldu=7), dict(dt=None), dict(lddt=7), dict(z=ODD), dict(ldz=7), dict(B=None),
    dict(ldB=15), dict(C=None), dict(ldC=15), dict(A=None), dict(A=P + 2), dict(D=P + 2),
    dict(bias=P + 2), dict(seq=P + 2), dict(slots=0)])
def test_scan_refusals(L, bad):
    s = scan(**bad)
    big = 1 << 40
    assert L.lirpa_scan_forward(s, None, None, P, 8, None, P, big, None) == lirpa.LIRPA_EINVAL
    assert L.lirpa_scan_step(s, P, P, P, 8, None) == lirpa.LIRPA_EINVAL
    assert L.lirpa_scan_backward(s, P, 8, P, P, 8, P, 8, P, 8, P, 16, P, 16, P, P, P, P, big,
                                 None) == lirpa.LIRPA_EINVAL


@pytest.mark.parametrize("bad,code", [
    (dict(state=P + 2), -1), (dict(state_out=P + 2), -1), (dict(y=None), -1), (dict(ldy=7), -1),
    (dict(kept=P + 8), -1), (dict(kept=P, state=P), -1), (dict(ws=None), -1), (dict(ws=P + 4), -1),
    (dict(ws_bytes=100), -2)])
def test_scan_forward_refusals(L, bad, code):
    a = dict(state=None, state_out=P, y=P, ldy=8, kept=None, ws=P, ws_bytes=1 << 40)
    a.update(bad)
    assert L.lirpa_scan_forward(scan(), *a.values(), None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dy=None), -1), (dict(lddy=7), -1), (dict(kept=None), -1), (dict(kept=P + 8), -1),
    (dict(du=None), -1), (dict(ddt=None), -1), (dict(dz=None), -1), (dict(lddz=1), -1),
    (dict(dB=None), -1), (dict(lddB=15), -1), (dict(dC=None), -1), (dict(dA=P + 2), -1),
    (dict(dD=P + 2), -1), (dict(dbias=P + 2), -1), (dict(ws=None), -1), (dict(ws_bytes=100), -2)])
def test_scan_backward_refusals(L, bad, code):
    a = dict(dy=P, lddy=8, kept=P, du=P, lddu=8, ddt=P, ldddt=8, dz=P, lddz=8, dB=P, lddB=16, dC=P,
             lddC=16, dA=P, dD=P, dbias=P, ws=P, ws_bytes=1 << 40)
    a.update(bad)
    assert L.lirpa_scan_backward(scan(), *a.values(), None) == code
    assert L.lirpa_scan_backward(scan(z=None), *{**a, "dz": P}.values(), None) == -1


def test_null_scan(L):
    assert L.lirpa_scan_forward(None, None, None, P, 8, None, P, 256, None) == lirpa.LIRPA_EINVAL
    assert "null" in lirpa.lirpa_last_error()


def test_no_rows(L):
    """Null buffers, as empty tensors have them."""
    none = scan(rows=0, u=None, dt=None, z=None, B=None, C=None, seq=None)
    assert L.lirpa_scan_forward(none, None, None, None, 0, None, None, 0, None) == 0
    assert L.lirpa_scan_step(none, None, None, None, 0, None) == 0
    for call in (L.lirpa_conv_forward, L.lirpa_conv_step):
        assert call(0, 0, 8, 4, None, 0, None, None, 0, None, 1, None, None, None, 0, None) == 0


def test_workspaces_hold_fewer_rows_too(L):
    rows = [*range(0, 700, 3), *range(700, 20000, 97), 1 << 17, 1 << 20, 1 << 30]
    for n, states in ((1, 1), (64, 16), (1001, 24), (4096, 16), (1 << 20, 64)):
        for backward in (0, 1):
            sizes = [L.lirpa_scan_workspace_bytes(r, n, states, backward) for r in rows]
            assert sizes[0] >= 256 and sizes == sorted(sizes)
        kept = [L.lirpa_scan_kept_bytes(r, n, states) for r in rows]
        assert kept[0] > 0 and kept == sorted(kept)
        sizes = [L.lirpa_conv_workspace_bytes(r, n, 4) for r in rows]
        assert sizes[0] >= 256 and sizes == sorted(sizes)
    for bad in ((-1, 8, 4), (4, 0, 4), (4, 8, 0), ((1 << 30) + 1, 8, 4)):
        assert L.lirpa_scan_workspace_bytes(*bad, 0) == 0
        assert L.lirpa_scan_kept_bytes(*bad) == 0
        assert L.lirpa_conv_workspace_bytes(*bad) == 0
    assert L.lirpa_scan_workspace_bytes(4, 8, 65, 0) == 0
    assert L.lirpa_scan_workspace_bytes(4, 8, 16, 2) == 0
    assert L.lirpa_conv_workspace_bytes(4, 8, 9) == 0


def test_sequences():
    seq = blocks.sequences([3, 0, 1], device="cpu")
    assert seq.tolist() == [0, 0, 0, 2] and seq.dtype == torch.int32
    assert blocks.sequences([2, 1], rows=5, slots=[7, 4], device="cpu").tolist() == [7, 7, 4, -1, -1]
    assert blocks.sequences([], rows=2, device="cpu").tolist() == [-1, -1]
    for bad in (dict(lengths=[2, -1]), dict(lengths=[2], rows=1), dict(lengths=[1, 1], slots=[3]),
                dict(lengths=[1, 1], slots=[3, 3]), dict(lengths=[1], slots=[-1])):
        with pytest.raises(ValueError):
            blocks.sequences(**bad, device="cpu")


def test_binding_refuses():
    x, w = torch.zeros(4, 8), torch.zeros(4, 8)
    with pytest.raises(ValueError, match="act"):
        blocks.CausalConv(w, act="relu")
    with pytest.raises(TypeError, match="CUDA"):
        blocks.CausalConv(w).forward(x)
    with pytest.raises(ValueError, match="two dimensions"):
        blocks.CausalConv(w).backward(x, x[0])
    s = blocks.SelectiveScan(torch.zeros(8, 2))
    with pytest.raises(TypeError, match="CUDA"):
        s.forward(x, x, x[:, :2], x[:, :2])
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        s.forward(x.double(), x, x[:, :2], x[:, :2])


def test_conv_workspace_is_what_a_call_writes(L):
    """Many rows are cut into strips of 32 - 2 (taps - 1) rows, each with a part of dw and dbias: no
    room for more, while few rows may be cut into strips of 8."""
    for n in (4096, 5000, 1 << 20):
        for taps in range(1, 9):
            longest = 32 - 2 * (taps - 1)
            for rows in (1 << 18, (1 << 20) + 7, 1 << 30):
                want = -(-rows // longest) * (taps + 1) * n * 4
                assert L.lirpa_conv_workspace_bytes(rows, n, taps) == want
    assert L.lirpa_conv_workspace_bytes(800, 64, 4) == 100 * 5 * 64 * 4
