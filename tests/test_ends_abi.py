"""Host-side checks of the embedding's and the log probabilities' entry points: sizes of their
workspaces, and bad arguments turned down before anything is enqueued (no call reaches a kernel)."""
import os

import pytest
import torch

from paper_2011_13824_amd import blocks, lirpa

P, Q = 0x10000, 0x20000  # stand for device pointers: only their alignment is looked at
ODD = P + 1


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(lirpa.LIB_PATH):
        import __graft_entry__
        __graft_entry__.build()
    return lirpa.load()


@pytest.mark.parametrize("bad", [
    dict(dtype=3), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(n=0), dict(n=(1 << 20) + 1),
    dict(vocab=0), dict(vocab=(1 << 20) + 1), dict(tokens=None), dict(tokens=P + 4),
    dict(table=None), dict(table=ODD), dict(ldt=7), dict(scale=float("nan")),
    dict(scale=float("inf")), dict(out=None), dict(ldo=1 << 22)])
def test_embed_forward_refusals(L, bad):
    a = dict(dtype=lirpa.BF16, rows=4, n=8, vocab=10, tokens=P, table=P, ldt=8, scale=1.0, out=P,
             ldo=8)
    a.update(bad)
    assert L.lirpa_embed_forward(*a.values(), None) == lirpa.LIRPA_EINVAL
    assert "lirpa_embed_forward" in lirpa.lirpa_last_error()


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=-1), -1), (dict(rows=-1), -1), (dict(n=0), -1), (dict(vocab=0), -1),
    (dict(tokens=None), -1), (dict(tokens=P + 2), -1), (dict(dout=None), -1), (dict(lddo=3), -1),
    (dict(scale=float("inf")), -1), (dict(base=ODD), -1), (dict(base=Q, ldb=7), -1),
    (dict(dtable=None), -1), (dict(ldd=7), -1), (dict(base=P, ldb=9), -1), (dict(ws=None), -1),
    (dict(ws=P + 8), -1), (dict(ws_bytes=1000), -2)])
def test_embed_backward_refusals(L, bad, code):
    a = dict(dtype=lirpa.F16, rows=4, n=8, vocab=10, tokens=P, dout=P, lddo=8, scale=1.0, base=None,
             ldb=0, dtable=P, ldd=8, ws=P, ws_bytes=1 << 30)
    a.update(bad)
    assert L.lirpa_embed_backward(*a.values(), None) == code


@pytest.mark.parametrize("bad,code", [
    (dict(dtype=5), -1), (dict(rows=-1), -1), (dict(n=0), -1), (dict(scale=0.0), -1),
    (dict(scale=-1.0), -1), (dict(scale=float("nan")), -1), (dict(scale=2.0 ** 101), -1), (dict(top=-1), -1), (dict(top=33), -1),
    (dict(logits=None), -1), (dict(logits=ODD), -1), (dict(ldl=7), -1), (dict(tokens=None), -1),
    (dict(tokens=P + 4), -1), (dict(logp=P + 2), -1), (dict(lse=P + 2), -1),
    (dict(entropy=P + 1), -1), (dict(top_logp=None), -1), (dict(top_tokens=None), -1),
    (dict(top_tokens=P + 4), -1), (dict(logp=None, lse=None, entropy=None, top=0), -1),
    (dict(ws=None), -1), (dict(ws=P + 4), -1), (dict(ws_bytes=100), -2)])
def test_logprob_forward_refusals(L, bad, code):
    a = dict(dtype=lirpa.BF16, rows=4, n=5000, logits=P, ldl=5000, scale=1.0, tokens=P, logp=P,
             lse=P, entropy=P, top=3, top_logp=P, top_tokens=P, ws=P, ws_bytes=1 << 30)
    a.update(bad)
    assert L.lirpa_logprob_forward(*a.values(), None) == code


@pytest.mark.parametrize("bad", [
    dict(dtype=5), dict(rows=-1), dict(n=0), dict(scale=0.0), dict(scale=float("inf")),
    dict(logits=None), dict(ldl=7),
    dict(tokens=None), dict(lse=None), dict(lse=P + 2), dict(entropy=None), dict(entropy=P + 2),
    dict(dlogp=P + 2), dict(dentropy=ODD), dict(dlogp=None, dentropy=None), dict(dlogits=None),
    dict(ldd=7), dict(dlogits=P, ldd=9)])
def test_logprob_backward_refusals(L, bad):
    a = dict(dtype=lirpa.F32, rows=4, n=8, logits=P, ldl=8, scale=1.0, tokens=P, lse=P, entropy=P,
             dlogp=P, dentropy=P, dlogits=Q, ldd=8)
    a.update(bad)
    assert L.lirpa_logprob_backward(*a.values(), None) == lirpa.LIRPA_EINVAL


def test_workspaces(L):
    for n in (1, 64, 1001, 4096, 1 << 20):
        last = 0
        for rows in (*range(300), *range(300, 9000, 31), 1 << 20, 1 << 30):
            need = L.lirpa_embed_workspace_bytes(rows, n)
            assert need >= max(last, 256)
            last = need
    for rows, n in ((-1, 8), (4, 0), ((1 << 30) + 1, 8), (4, (1 << 20) + 1)):
        assert L.lirpa_embed_workspace_bytes(rows, n) == 0
        assert L.lirpa_logprob_workspace_bytes(rows, n, 0) == 0
    assert L.lirpa_logprob_workspace_bytes(4, 8, 33) == 0
    assert L.lirpa_logprob_workspace_bytes(4, 8, -1) == 0
    for n in (1, 2048, 2049, 1 << 20):
        for top in (0, 32):
            sizes = [L.lirpa_logprob_workspace_bytes(r, n, top) for r in (0, 1, 64, 1024, 1 << 30)]
            assert sizes[0] > 0 and sizes == sorted(sizes)


def test_no_rows(L):
    """Null buffers, as empty tensors have them."""
    assert L.lirpa_embed_forward(0, 0, 8, 10, None, None, 0, 1.0, None, 0, None) == 0
    assert L.lirpa_logprob_forward(0, 0, 8, None, 0, 1.0, None, None, None, None, 0, None, None,
                                   None, 0, None) == 0
    assert L.lirpa_logprob_backward(0, 0, 8, None, 0, 1.0, None, None, None, None, None, None, 0,
                                    None) == 0


def test_binding_refuses():
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    with pytest.raises(TypeError, match="CUDA"):
        blocks.Embedding(x).forward(t)
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        blocks.Embedding(x.double()).forward(t)
    with pytest.raises(ValueError, match="two dimensions"):
        blocks.Embedding(x[0]).forward(t)
    with pytest.raises(ValueError, match="out must be"):
        blocks.Embedding(x).backward(t, x, out=x[:, :4])
    with pytest.raises(TypeError, match="CUDA"):
        blocks.LogProbs().forward(x, t)
    with pytest.raises(ValueError, match="two dimensions"):
        blocks.LogProbs().forward(x[0], t)
    with pytest.raises(TypeError, match="CUDA"):
        blocks.LogProbs().backward(x, t, torch.zeros(4), dlogp=torch.zeros(4))


@pytest.mark.parametrize("top", [-1, 33])
def test_more_alternatives_than_there_are_places(top):
    with pytest.raises(ValueError, match="top"):
        blocks.LogProbs(top=top)
