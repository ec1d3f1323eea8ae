"""The feed-forward block's calls where their contract is easily broken: buffers that are shared,
ends of the types' ranges, batches that do not belong together, many rows."""
import warnings

import pytest
import torch

from .test_gpu_blocks import UNIT, backward64, check, forward64

pytestmark = pytest.mark.gpu

TYPES = [torch.float32, torch.bfloat16, torch.float16]


def ids(t):
    return str(t).replace("torch.", "")


@pytest.fixture(scope="module")
def B():
    from paper_2011_13824_amd import blocks
    return blocks


@pytest.fixture(scope="module")
def lirpa():
    from paper_2011_13824_amd import lirpa
    return lirpa


def rand(seed, *shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)


# ---------------------------------------------------------------------------------------------
# Shared buffers
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("n", [200, 4095, 5000, 16384, 16385, 17000, 40000])
@pytest.mark.parametrize("where", ["dy", "dsum"])
def test_norm_gradient_in_place_with_weights(lirpa, B, dtype, n, where):
    """dh in the buffer of dy or of dsum is what it is in one of its own, and so is dw."""
    rows = 7
    dy, h, ds = (rand(s, rows, n, dtype=dtype) for s in (1, 2, 3))
    w = rand(4, n, dtype=dtype)
    rstd = torch.rsqrt(h.float().square().mean(1) + 1e-5)
    dh, dw = B.Norm(w).backward(dy, h, rstd, ds)
    need = lirpa.lirpa_norm_workspace_bytes(rows, n)
    ws, dw2 = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty_like(dw)
    to = dy if where == "dy" else ds
    lirpa.lirpa_norm_backward(dy, ds, h, w, rstd, to, dw2, ws, need)
    assert torch.equal(to, dh)
    assert torch.equal(dw2, dw)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("D,F", [(1024, 2752), (256, 4288)])
def test_one_workspace_for_all_batches(lirpa, B, dtype, D, F):
    """A workspace for the largest batch, full of NaN, serves every smaller one, and what a call
    leaves there is not read by the next."""
    most = 800
    W = [rand(s, *shape, dtype=dtype, scale=0.05)
         for s, shape in ((1, (F, D)), (2, (F, D)), (3, (D, F)))]
    ffn = B.FeedForward(*W)
    needs = [lirpa.lirpa_ffn_workspace_bytes(ffn.block, most, b) for b in (0, 1)]
    ws = torch.full((max(needs) // 4 + 1,), float("nan"), device="cuda").view(torch.uint8)
    for rows in (800, 769, 768, 357, 356, 129, 65, 9, 1):
        x, dout = rand(rows, rows, D, dtype=dtype), rand(rows + 1, rows, D, dtype=dtype)
        want, kept = ffn.forward(x, keep=0)
        grads = ffn.backward(dout, kept)
        out, g, u = torch.empty_like(x), torch.empty_like(kept.g), torch.empty_like(kept.u)
        lirpa.lirpa_ffn_forward(ffn.block, x, out, lirpa.KEEP_FULL, g, u, ws, needs[0])
        assert torch.equal(out, want) and torch.equal(g, kept.g) and torch.equal(u, kept.u), rows
        got = [torch.empty_like(t) for t in (x, *W)]
        lirpa.lirpa_ffn_backward(ffn.block, dout, lirpa.KEEP_FULL, x, g, u, *got, ws, needs[1])
        for name, t in zip(("dx", "dWg", "dWu", "dWd"), got):
            assert torch.equal(t, grads[name]), (rows, name)


# ---------------------------------------------------------------------------------------------
# What does not belong together
# ---------------------------------------------------------------------------------------------
def test_packed_activations_of_another_matrix_are_refused(B):
    """Larger ones too: where the scales lie follows from the matrix."""
    D, F = 64, 96
    ffn = B.FeedForward(rand(1, F, D), rand(2, F, D), rand(3, D, F))
    x, dout = rand(4, 40, D), rand(5, 40, D)
    for x8 in (B.Q8.pack(rand(6, 41, D)), B.Q8.pack(rand(6, 39, D)), B.Q8.pack(rand(6, 40, D + 1)),
               B.Q8.pack(rand(6, 41, D)).buf):
        with pytest.raises(ValueError, match="x8"):
            ffn.forward(x, keep=8, x8=x8)
    for keep in (8, 0):
        _, kept = ffn.forward(x, keep=keep)
        for rows in (39, 41):
            with pytest.raises(ValueError, match="40 rows were kept"):
                ffn.backward(rand(7, rows, D), kept)
        ffn.backward(dout, kept)
    other = B.Q8.pack(rand(8, 41, F))
    _, kept = ffn.forward(x, keep=8)
    for x8, g, u in ((kept.x, other, kept.u), (kept.x, kept.g, other),
                     (B.Q8.pack(rand(9, 41, D)), kept.g, kept.u),
                     (kept.x, other.buf, kept.u), (kept.g, kept.g, kept.u)):
        with pytest.raises(ValueError, match="must"):
            ffn.backward(dout, B.Kept(8, 40, x8, g, u))
    raw = ffn.backward(dout, B.Kept(8, 40, kept.x.buf, kept.g.buf, kept.u.buf))
    want = ffn.backward(dout, kept)
    assert all(torch.equal(raw[k], want[k]) for k in want)
    with pytest.raises(ValueError, match="bytes"):
        B.Q8(40, D, other.buf).values()


# ---------------------------------------------------------------------------------------------
# Ends of the types' ranges
# ---------------------------------------------------------------------------------------------
def test_q8_f16_keeps_finite_values_finite(B):
    """Magnitudes from 65024 on are 64 * 2^10 in 8 bits: past f16's range, read as its largest."""
    f16 = torch.float16
    for top in (64992.0, 65024.0, 65056.0, 65504.0):
        for sign in (1, -1):
            x = rand(1, 3, 70, dtype=f16)
            x[1, 37] = sign * top
            q = B.Q8.pack(x)
            v = q.values(f16)
            assert torch.isfinite(v).all()
            assert abs(v[1, 37].item() - sign * top) <= 512  # half a step of 2^10
            wide = q.values(torch.float32)
            assert torch.equal(v, wide.clamp(-65504, 65504).to(f16))
    x = rand(1, 3, 70, dtype=f16)
    x[1, 37] = float("inf")
    v = B.Q8.pack(x).values(f16)
    assert torch.isnan(v[1, 32:64]).all() and torch.isfinite(v[1, :32]).all()


def test_ffn_gradients_from_f16_activations_at_the_end_of_the_range(B):
    """A finite x near 65504, kept in 8 bits, leaves finite weight gradients: those of its value."""
    rows, D, F = 40, 72, 104
    dt = torch.float16
    W = [rand(s, *shape, dtype=dt, scale=1e-3)
         for s, shape in ((1, (F, D)), (2, (F, D)), (3, (D, F)))]
    x, dout = rand(4, rows, D, dtype=dt), rand(5, rows, D, dtype=dt, scale=1e-3)
    x[3, 7], x[9, 70] = 65504.0, -65300.0
    kept = B.Kept(8, rows, *(B.Q8.pack(t) for t in (x, rand(6, rows, F), rand(7, rows, F))))
    got = B.FeedForward(*W, "silu").backward(dout, kept)
    vx, g, u = (t.values().double() for t in (kept.x, kept.g, kept.u))
    vx = vx.clamp(-65504, 65504)
    p = torch.sigmoid(g)
    da = dout.double() @ W[2].double()
    dg, du = da * u * p * (1 + g * (1 - p)), da * g * p
    unit = 2.0 ** -11
    for name, d in (("dWg", dg), ("dWu", du)):
        want = d.T @ vx
        # dg and du are rounded to f16 (2^-25 at the least), as is the result; the rest is under that
        tol = (2 * unit * d.abs() + 2.0 ** -24).T @ vx.abs() + unit * want.abs() + 2.0 ** -24
        assert torch.isfinite(got[name]).all()
        assert ((got[name].double() - want).abs() <= tol).all(), name


E = 2.0 ** -24


def test_ffn_f32_finite_at_the_end_of_the_range(B):
    """Finite floats over bf16's largest, 3.3895e38, are summed as what they are."""
    rows, D, F = 90, 72, 104
    x, dout = rand(1, rows, D), rand(2, rows, D, scale=1e-25)
    W = [rand(s, *shape, scale=0.1) for s, shape in ((3, (F, D)), (4, (F, D)), (5, (D, F)))]
    for i, top in ((3, 3.4e38), (70, -3.4028e38)):
        x[i, 5] = top
    for w in W[:2]:
        w[:, 5] *= 1e-30
    ffn = B.FeedForward(*W, "relu")
    out, kept = ffn.forward(x, keep=0)
    x64 = x.double()
    for got, w in ((kept.g, W[0]), (kept.u, W[1])):
        want = x64 @ w.double().T
        tol = (D + 8) * E * (x64.abs() @ w.double().abs().T) + E * want.abs()
        assert ((got.double() - want).abs() <= tol).all()
    assert torch.isfinite(out).all()
    g, u = rand(6, rows, F), rand(7, rows, F)
    got = ffn.backward(dout, B.Kept(0, rows, x, g, u))
    d64, w64, g64, u64 = dout.double(), W[2].double(), g.double(), u.double()
    da, tda = d64 @ w64, (D + 8) * E * (d64.abs() @ w64.abs())
    for name, by in (("dWg", u64 * (g64 > 0)), ("dWu", g64.clamp(min=0))):
        d, td = da * by, tda * by.abs() + 8 * E * (da * by).abs()
        want = d.T @ x64
        tol = (td + (rows + 8) * E * d.abs()).T @ x64.abs() + E * want.abs()
        assert ((got[name].double() - want).abs() <= tol).all(), name


def test_ffn_f32_at_the_other_end(B):
    """Under 2^-109 the parts of a float under 2^-126 may be lost: that much of it, no more."""
    rows, D, F = 90, 72, 104
    W = [rand(s, *shape) for s, shape in ((3, (F, D)), (4, (F, D)), (5, (D, F)))]
    for scale in (1e-30, 1e-34, 1e-37, 1e-39):
        x = rand(1, rows, D, scale=scale)
        kept = B.FeedForward(*W, "relu").forward(x, keep=0)[1]
        x64, w64 = x.double(), W[0].double()
        want, size = x64 @ w64.T, x64.abs() @ w64.abs().T
        tol = (D + 8) * E * size + 2.0 ** -125 * (w64.abs().sum(1) + 1)
        assert ((kept.g.double() - want).abs() <= tol).all(), scale


@pytest.mark.parametrize("rows", [8, 64, 65])
def test_ffn_f32_infinities_stay_infinite_or_nan(B, rows):
    W = [rand(s, *shape, scale=0.1) for s, shape in ((3, (104, 72)), (4, (104, 72)), (5, (72, 104)))]
    W[0][7], W[1][9] = 1.0, 0.5  # one part alone
    x = rand(1, rows, 72)
    ffn = B.FeedForward(*W, "silu")
    clean, kept0 = ffn.forward(x, keep=0)
    x[5, 11] = float("inf")
    for keep in (None, 0):
        out = ffn.forward(x, keep=keep)
        out, kept = out if keep == 0 else (out, None)
        others = [r for r in range(rows) if r != 5]
        assert not torch.isfinite(out[5]).any()
        if keep == 0:
            assert torch.equal(out[others], clean[others])
            assert not torch.isfinite(kept.g[5]).any() and not torch.isfinite(kept.u[5]).any()
            assert torch.equal(kept.g[others], kept0.g[others])


# ---------------------------------------------------------------------------------------------
# Launches
# ---------------------------------------------------------------------------------------------
@pytest.mark.parametrize("rows", [8192, 8193])
def test_ffn_gradients_share_a_launch(lirpa, B, rows):
    """Also where dx's tiles fill the CUs twice and leave a few over: by itself those would leave
    the rest idle."""
    D, F, dt = 4096, 1024, torch.bfloat16
    ffn = B.FeedForward(rand(1, F, D, dtype=dt), rand(2, F, D, dtype=dt), rand(3, D, F, dtype=dt))
    x = rand(4, rows, D, dtype=dt)
    _, kept = ffn.forward(x, keep=8)
    lirpa.lirpa_timing_begin()
    ffn.backward(x, kept)
    assert lirpa.lirpa_timing_end()["ffn_grads"][1] == 1


# ---------------------------------------------------------------------------------------------
# Weights that move
# ---------------------------------------------------------------------------------------------
def test_ffn_reads_the_weights_as_they_are(B):
    """After ``w.data = other``, of any layout or type, a call is that of a block made anew."""
    D, F, rows = 72, 104, 90
    W = [rand(s, *shape, scale=0.1) for s, shape in ((1, (F, D)), (2, (F, D)), (3, (D, F)))]
    ffn = B.FeedForward(*W, "gelu")
    x, dout = rand(4, rows, D), rand(5, rows, D)
    ffn.backward(dout, ffn.forward(x, keep=8)[1])
    held = [w.data for w in W]  # the old storage stays alive
    for k, (pad, dtype) in enumerate([(0, torch.float32), (3, torch.float32), (0, torch.bfloat16),
                                      (5, torch.bfloat16), (8, torch.float16)]):
        for i, w in enumerate(W):
            r, n = held[i].shape
            w.data = rand(10 * k + i, r, n + pad, dtype=dtype, scale=0.1)[:, :n]
        new = B.FeedForward(*(w.data for w in W), "gelu")
        xt, dt = x.to(dtype), dout.to(dtype)
        assert torch.equal(ffn.forward(xt[:3]), new.forward(xt[:3])), k
        (out, kept), (want, nkept) = ffn.forward(xt, keep=8), new.forward(xt, keep=8)
        assert torch.equal(out, want), k
        got, grads = ffn.backward(dt, kept), new.backward(dt, nkept)
        assert all(torch.equal(got[n], grads[n]) for n in grads), k


# ---------------------------------------------------------------------------------------------
# Autograd
# ---------------------------------------------------------------------------------------------
def test_a_lost_gradient_is_warned_of(B):
    D, F = 24, 40
    x, w = rand(1, 5, D), rand(2, D)
    W = [rand(s, *shape) for s, shape in ((3, (F, D)), (4, (F, D)), (5, (D, F)))]

    def forward():
        return B.Norm(w).forward(x, x), B.FeedForward(*W).forward(x)

    with warnings.catch_warnings():
        warnings.simplefilter("error")
        forward()
        for t in (x, w, W[1]):
            t.requires_grad_()
            with torch.no_grad():
                forward()
            t.requires_grad_(False)
    for t, call in ((x, lambda: B.Norm(w).forward(x)), (w, lambda: B.Norm(w).forward(x)),
                    (x, lambda: B.FeedForward(*W).forward(x)),
                    (W[2], lambda: B.FeedForward(*W).forward(x, keep=8))):
        t.requires_grad_()
        with pytest.warns(UserWarning, match="autograd does not record"):
            call()
        t.requires_grad_(False)


def test_what_is_no_tensor_is_a_type_error(B):
    x = rand(1, 5, 24)
    ffn = B.FeedForward(rand(2, 40, 24), rand(3, 40, 24), rand(4, 24, 40))
    for call in (lambda: B.Norm([1.0] * 24).forward(x),
                 lambda: B.Norm(rand(5, 24)).forward(x, x.tolist()),
                 lambda: B.Norm(rand(5, 24)).forward(x.cpu().numpy()),
                 lambda: ffn.forward(x.cpu().numpy())):
        with pytest.raises(TypeError):
            call()


# ---------------------------------------------------------------------------------------------
# Rows
# ---------------------------------------------------------------------------------------------
def test_one_row_has_no_row_distance(B):
    """The last token of a long sequence: a row whose tensor's stride passes 2^22."""
    D, F, dt = 64, 96, torch.bfloat16
    seq = rand(1, 1, (1 << 22) // D + 3, D, dtype=dt)
    x = seq[:, -1]
    assert x.shape == (1, D) and x.stride(0) >= 1 << 22
    same = x.clone(memory_format=torch.contiguous_format)
    ffn = B.FeedForward(rand(2, F, D, dtype=dt), rand(3, F, D, dtype=dt), rand(4, D, F, dtype=dt))
    norm = B.Norm(rand(5, D, dtype=dt))
    assert torch.equal(ffn.forward(x), ffn.forward(same))
    n, want = norm.forward(x, x, want8=True), norm.forward(same, same, want8=True)
    assert torch.equal(n.y, want.y) and torch.equal(n.sum, want.sum)
    assert torch.equal(n.y8.buf, want.y8.buf)
    assert torch.equal(B.Q8.pack(x).buf, B.Q8.pack(same).buf)
    (_, kept), (_, nkept) = ffn.forward(x, keep=0), ffn.forward(same, keep=0)
    got, grads = ffn.backward(x, kept), ffn.backward(same, nkept)
    assert all(torch.equal(got[k], grads[k]) for k in grads)


def test_norm_of_more_rows_than_a_launch_takes(B):
    """2^26 rows of a wave each are 2^32 threads."""
    rows = (1 << 26) + 5
    x = rand(1, rows, 1, dtype=torch.bfloat16)
    w = torch.full((1,), 1.5, dtype=torch.bfloat16, device="cuda")
    got = B.Norm(w).forward(x, x, want8=True)
    h = 2 * x.float()
    rstd = torch.rsqrt(h[:, 0].square() + 1e-5)
    assert ((got.rstd - rstd).abs() <= 16 * E * rstd).all()
    assert torch.equal(got.sum, h.to(x.dtype))
    del rstd
    y = h * got.rstd[:, None] * 1.5
    assert ((got.y.float() - y).abs() <= 2.0 ** -7 * y.abs()).all()
    # the packed y is within half a step, its scale the least one
    v = got.y8.values()
    assert ((v - y).abs() <= y.abs() / 126).all()
    dh, dw = B.Norm(w).backward(x, got.sum, got.rstd)
    assert torch.isfinite(dh[-9:]).all() and torch.isfinite(dw).all()


def test_q8_of_the_most_rows(B):
    """2^30 rows of one group each are 2^32 threads; the scales lie 2^35 bytes into the buffer."""
    rows = 1 << 30
    x = torch.arange(rows, dtype=torch.int32, device="cuda").remainder_(251).sub_(125)
    x = x.to(torch.bfloat16).view(rows, 1)  # one value a group: exact in 8 bits
    q = B.Q8.pack(x)
    assert q.buf.numel() == rows * 33
    assert torch.equal(q.values(torch.bfloat16), x)


@pytest.mark.parametrize("keep", [8, 0])
def test_ffn_of_more_values_than_32_bits_count(B, keep):
    """Projections of 2^31 and more values: the last rows, and the weights' gradients, to which they
    alone contribute, against 64 bits."""
    D, F, rows, last, dt = 64, 2112, 1 << 20, 90, torch.bfloat16
    W = [rand(s, *shape, dtype=dt, scale=0.1)
         for s, shape in ((1, (F, D)), (2, (F, D)), (3, (D, F)))]
    ffn = B.FeedForward(*W)
    x, dout = rand(4, rows, D, dtype=dt), torch.zeros(rows, D, dtype=dt, device="cuda")
    dout[-last:] = rand(5, last, D, dtype=dt)
    got, kept = ffn.forward(x, keep=keep)
    out, tol, g, tg, u, tu = forward64(x[-last:], W, "silu", UNIT[dt])
    check(got[-last:], out, tol + 1e-30, "out")
    if keep == 0:
        ends = [t[-last:] for t in (x, kept.g, kept.u)]
        check(ends[1], g, tg + UNIT[dt] * g.abs(), "g")
        check(ends[2], u, tu + UNIT[dt] * u.abs(), "u")
    else:
        ends = [t.values()[-last:] for t in (kept.x, kept.g, kept.u)]
    grads = ffn.backward(dout, kept)
    assert (grads["dx"][:-last] == 0).all()
    grads["dx"] = grads["dx"][-last:]
    want, tol = backward64(dout[-last:], ends[0], ends[1].double(), ends[2].double(), W, "silu",
                           UNIT[dt])
    for name in want:
        check(grads[name], want[name], tol[name] + 1e-30, name)
