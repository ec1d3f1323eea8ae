"""Causal convolution and selective scan against plain implementations in 64 bits.

Tolerances are bounds, not measurements.  With u the rounding unit of the type and e = 2^-24 that of
32 bits, every elementary step is off by its own rounding and by what its arguments are off: the plain
implementation carries a bound of the error along with the value, through the same recurrence.  What
it takes for the steps:

* e^-|x| is off by (2 |x| + 2) e of itself, log(1 + e^x) by that and 10 e more (a reciprocal, the
  series, the sum), the sigmoid by that and 4 e;
* e^(delta A) by |delta A| times what delta is off and 3 e more (A in powers of two, the product,
  both of |delta A|), and 2 e;
* a sum of K terms by (K + 4) e times the sum of their magnitudes;
* joining chunks multiplies their decays, whose exponents are sums of delta: one more step each.
"""
import pytest
import torch

from .test_gpu_blocks import E, TINY, TYPES, UNIT, check, gen_of, ids, rand

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2011_13824_amd import blocks
    return blocks


@pytest.fixture(scope="module")
def lirpa():
    from paper_2011_13824_amd import lirpa
    return lirpa


def runs_of(seq, slots=1 << 31):
    """[(first row, rows, slot)] of the sequences; padding has none."""
    out, seq = [], seq.tolist()
    t = 0
    while t < len(seq):
        end = t
        while end < len(seq) and seq[end] == seq[t]:
            end += 1
        if 0 <= seq[t] < slots:
            out.append((t, end - t, seq[t]))
        t = end
    return out


# ---------------------------------------------------------------------------------------------
# Convolution
# ---------------------------------------------------------------------------------------------
def gate_of(pre, act):
    """(act(pre), its slope) in 64 bits"""
    if act == "linear":
        return pre, torch.ones_like(pre)
    s = torch.sigmoid(pre)
    return pre * s, s * (1 + pre * (1 - s))


def plain_conv(x, w, bias, act, runs, state=None, dy=None):
    """Outputs and their bounds, the states behind the sequences, gradients and their bounds."""
    rows, n = x.shape
    taps = w.shape[0]
    x, w = x.double(), w.double()
    b = bias.double() if bias is not None else torch.zeros(n, dtype=torch.float64, device="cuda")
    y, ty, dx, tx = (torch.zeros(rows, n, dtype=torch.float64, device="cuda") for _ in range(4))
    dw, tw = (torch.zeros(taps, n, dtype=torch.float64, device="cuda") for _ in range(2))
    db, tb = (torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2))
    last = {}
    for a, r, slot in runs:
        front = state[slot].double() if state is not None else x.new_zeros(taps - 1, n)
        p = torch.cat([front, x[a:a + r]])
        last[slot] = p[r:]
        pre, size = b.expand(r, n).clone(), b.abs().expand(r, n).clone()
        for k in range(taps):
            pre += w[k] * p[k:k + r]
            size += (w[k] * p[k:k + r]).abs()
        off = (taps + 5) * E * size
        y[a:a + r], slope = gate_of(pre, act)
        ty[a:a + r] = 1.1 * off + (8 + 3 * pre.abs()) * E * y[a:a + r].abs()
        if dy is None:
            continue
        d = dy[a:a + r].double() * slope
        td = dy[a:a + r].double().abs() * (0.5 * off + (16 + 4 * pre.abs()) * E * (1 + pre.abs()))
        zeros = d.new_zeros(taps - 1, n)
        ahead, tahead = torch.cat([d, zeros]), torch.cat([td, zeros])
        for k in range(taps):
            j = taps - 1 - k
            dx[a:a + r] += w[k] * ahead[j:j + r]
            tx[a:a + r] += w[k].abs() * (tahead[j:j + r] + (taps + 4) * E * ahead[j:j + r].abs())
            dw[k] += (d * p[k:k + r]).sum(0)
            tw[k] += (p[k:k + r].abs() * (td + (rows + 4) * E * d.abs())).sum(0)
        db += d.sum(0)
        tb += (td + (rows + 4) * E * d.abs()).sum(0)
    return dict(y=(y, ty), dx=(dx, tx), dw=(dw, tw), dbias=(db, tb)), last


def layout(g, rows, kind):
    """seq, or None"""
    if kind == "one":
        return None
    if kind == "ones":
        return torch.randperm(rows, generator=g, device="cuda").to(torch.int32)
    seq = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
    if kind == "padding":
        return seq
    # ragged: lengths of 1, of a span, of a chunk, with padding between and behind
    t, slot, sizes = 0, 3, [1, 2, 16, 15, 64, 48, 1, 90, 129, 7]
    for i in range(1000):
        size = sizes[i % len(sizes)]
        if t + size > rows - rows // 20:
            break
        seq[t:t + size] = slot
        t += size
        slot += 2
        if i % 3 == 2:
            seq[t:t + 2] = -1 - i
            t += 2
    return seq


def within(got, pair, dtype, what):
    want, tol = pair
    check(got, want, tol + (UNIT[dtype] + E) * want.abs() + TINY[dtype], what)


CONV_SHAPES = [(1, 1, 4, "one"), (2, 9, 4, "one"), (3, 64, 3, "one"), (70, 33, 2, "ragged"),
               (300, 129, 4, "ragged"), (37, 40, 8, "ragged"), (64, 24, 1, "ragged"),
               (50, 16, 5, "ones"), (900, 1024, 4, "ragged"), (5, 8, 6, "padding"),
               (4500, 257, 4, "ragged"), (2100, 2056, 4, "one"), (33, 8, 7, "one")]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,n,taps,kind", CONV_SHAPES)
@pytest.mark.parametrize("act,bias,pad", [("silu", True, 0), ("linear", False, 3)])
def test_conv(B, dtype, rows, n, taps, kind, act, bias, pad):
    g = gen_of(rows + n + taps)
    x, dy = (rand(g, rows, n, dtype=dtype, pad=pad, shift=1 if pad else 0) for _ in range(2))
    w = rand(g, taps, n, dtype=dtype)
    b = rand(g, 1, n, dtype=dtype)[0] if bias else None
    seq = layout(g, rows, kind)
    runs = [(0, rows, 0)] if seq is None else runs_of(seq)
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for a, r, _ in runs:
        inside[a:a + r] = True
    x[~inside], dy[~inside] = float("nan"), float("nan")  # of no account
    op = B.CausalConv(w, b, act)
    want, _ = plain_conv(x, w, b, act, runs, dy=dy)
    y = op.forward(x, seq)
    within(y, want["y"], dtype, "y")
    grads = op.backward(dy, x, seq)
    assert set(grads) == ({"dx", "dw", "dbias"} if bias else {"dx", "dw"})
    for k, v in grads.items():
        within(v, want[k], dtype, k)
    for t in (y, grads["dx"]):
        assert (t[~inside] == 0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("taps", [2, 4, 8])
@pytest.mark.parametrize("kind", ["one", "ragged", "ones"])
@pytest.mark.parametrize("same", [True, False])
def test_conv_states(B, dtype, taps, kind, same):
    """From states to states, in place or not; slots that are not named keep what they hold."""
    g = gen_of(taps)
    rows, n = 500, 43
    x, w = rand(g, rows, n, dtype=dtype), rand(g, taps, n, dtype=dtype)
    seq = layout(g, rows, kind)
    slots = 1 if seq is None else int(seq.max()) + 3
    if kind == "ragged":
        slots -= 5  # the last sequences have no slot: they are padding
    state = rand(g, slots * (taps - 1), n, dtype=dtype).view(slots, taps - 1, n).clone()
    runs = [(0, rows, 0)] if seq is None else runs_of(seq, slots)
    op = B.CausalConv(w)
    want, last = plain_conv(x, w, None, "silu", runs, state)
    before = state.clone()
    out = state if same else torch.full_like(state, 7.0)
    y = op.forward(x, seq, state, out)
    within(y, want["y"], dtype, "y")
    for s in range(slots):
        if s in last:
            assert torch.equal(out[s].double(), last[s]), s
        else:
            assert torch.equal(out[s], before[s] if same else torch.full_like(before[s], 7.0))
    if not same:
        assert torch.equal(state, before)
    if kind == "ones":  # single rows are a step
        again = before.clone()
        y2 = op.step(x, again, seq, again)
        assert torch.equal(y2, y) and torch.equal(again[seq.long()], out[seq.long()])
    assert torch.equal(op.forward(x, seq, before), y)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
def test_conv_in_parts(B, dtype):
    """A sequence in parts, one row at a time at its end, is the sequence."""
    g = gen_of(9)
    x, w, b = rand(g, 200, 30, dtype=dtype), rand(g, 4, 30, dtype=dtype), rand(g, 1, 30, dtype=dtype)
    op = B.CausalConv(w, b[0])
    whole = op.forward(x)
    state = torch.full((1, 3, 30), float("nan"), dtype=dtype, device="cuda")
    parts = [op.forward(x[:1], state_out=state)]
    for a, e in ((1, 3), (3, 70), (70, 190)):
        parts.append(op.forward(x[a:e], state=state, state_out=state))
    for t in range(190, 200):
        parts.append(op.step(x[t:t + 1], state, state_out=state))
    assert torch.equal(torch.cat(parts), whole)


# ---------------------------------------------------------------------------------------------
# Scan
# ---------------------------------------------------------------------------------------------
def plain_scan(u, dt, Bm, Cm, z, A, D, bias, runs, state=None, dy=None):
    """Values with their bounds, by the recurrences; the states behind the sequences."""
    d64 = dict(dtype=torch.float64, device="cuda")
    rows, n = u.shape
    N = A.shape[1]
    u, dt, Bm, Cm, A = (t.double() for t in (u, dt, Bm, Cm, A))
    D = D.double() if D is not None else torch.zeros(n, **d64)
    x = dt + (bias.double() if bias is not None else 0)
    delta = torch.logaddexp(x, torch.zeros_like(x))
    k = (2 * x.abs() + 14) * E + x.abs() * E  # of delta; dt + bias is rounded too
    slope = torch.sigmoid(x)
    out = {name: (torch.zeros(rows, n, **d64), torch.zeros(rows, n, **d64))
           for name in ("y", "du", "ddt", "dz")}
    for name in ("dB", "dC"):
        out[name] = torch.zeros(rows, N, **d64), torch.zeros(rows, N, **d64)
    out["dA"] = torch.zeros(n, N, **d64), torch.zeros(n, N, **d64)
    for name in ("dD", "dbias"):
        out[name] = torch.zeros(n, **d64), torch.zeros(n, **d64)
    last = {}

    def put(name, at, value, bound):
        out[name][0][at], out[name][1][at] = value, bound

    def add(name, value, bound):
        out[name][0].add_(value)
        out[name][1].add_(bound)

    for a, r, slot in runs:
        at = slice(a, a + r)
        s, us, ks = delta[at], u[at], k[at]
        arg = s[:, :, None] * A
        decay = torch.exp(arg)
        off = arg.abs() * (ks[:, :, None] + 6 * E) + 4 * E  # of the decay, relative; two of a chunk
        b = (s * us)[:, :, None] * Bm[at][:, None, :]
        tb = b.abs() * (ks[:, :, None] + 4 * E)
        h, th, size = (torch.zeros(r, n, N, **d64) for _ in range(3))
        first = state[slot].double() if state is not None else torch.zeros(n, N, **d64)
        now, tnow, mag = first, torch.zeros(n, N, **d64), first.abs()
        for t in range(r):
            tnow = decay[t] * (tnow + off[t] * mag) + tb[t]
            now = decay[t] * now + b[t]
            mag = decay[t] * mag + b[t].abs()
            tnow = tnow + 3 * E * mag
            h[t], th[t], size[t] = now, tnow, mag
        last[slot] = now, tnow
        C = Cm[at][:, None, :]
        v = (h * C).sum(2) + D * us
        tv = (C.abs() * (th + (N + 6) * E * size)).sum(2) + 3 * E * (D * us).abs() + 2 * E * v.abs()
        if z is not None:
            zs = z[at].double()
            sig = torch.sigmoid(zs)
            gate, gslope = zs * sig, sig * (1 + zs * (1 - sig))
            tz = (8 + 3 * zs.abs()) * E
        else:
            gate, gslope, tz, zs = 1.0, 0.0, torch.zeros_like(v), torch.zeros_like(v)
        put("y", at, v * gate, tv * (abs(gate) + tz) + tz * (v * gate).abs())
        if dy is None:
            continue
        dys = dy[at].double()
        p = dys * gate
        tp = p.abs() * tz
        put("dz", at, dys * v * gslope,
            dys.abs() * (1.2 * tv + v.abs() * (16 + 4 * zs.abs()) * E * (1 + zs.abs())))
        g, tg, gsize = (torch.zeros(r, n, N, **d64) for _ in range(3))
        now, tnow, mag = (torch.zeros(n, N, **d64) for _ in range(3))
        for t in range(r - 1, -1, -1):
            if t + 1 < r:
                tnow = decay[t + 1] * (tnow + off[t + 1] * mag)
                now, mag = decay[t + 1] * now, decay[t + 1] * mag
            now = now + C[t] * p[t][:, None]
            mag = mag + (C[t] * p[t][:, None]).abs()
            tnow = tnow + C[t].abs() * tp[t][:, None] + 3 * E * mag
            g[t], tg[t], gsize[t] = now, tnow, mag
        before, tbefore, bsize = (torch.zeros_like(h) for _ in range(3))
        before[1:], tbefore[1:], bsize[1:] = h[:-1], th[:-1], size[:-1]
        e = g * decay * before
        esize = gsize * decay * bsize
        te = decay * (tg * bsize + gsize * tbefore) + esize * (off + 4 * E)
        Bs = Bm[at][:, None, :]
        gB, tgB = (g * Bs).sum(2), (Bs.abs() * (tg + (N + 6) * E * gsize)).sum(2)
        gBsize = (Bs.abs() * gsize).sum(2)
        put("du", at, s * gB + D * p, s * (tgB + gBsize * (ks + 3 * E)) + D.abs() * (tp + 3 * E * p.abs()))
        dd = (e * A).sum(2) + us * gB
        tdd = (A.abs() * (te + (N + 6) * E * esize)).sum(2) + us.abs() * (tgB + 3 * E * gBsize)
        dsize = (A.abs() * esize).sum(2) + us.abs() * gBsize
        put("ddt", at, dd * slope[at],
            slope[at] * (tdd + dsize * (8 + 3 * x[at].abs()) * E))
        du_ = (s * us)[:, :, None]
        put("dB", at, (g * du_).sum(1),
            ((tg + gsize * (ks[:, :, None] + (n + 6) * E)) * du_.abs()).sum(1))
        put("dC", at, (p[:, :, None] * h).sum(1),
            (tp[:, :, None] * size + p.abs()[:, :, None] * (th + (n + 6) * E * size)).sum(1))
        add("dA", (e * s[:, :, None]).sum(0),
            (s[:, :, None] * (te + esize * (ks[:, :, None] + (rows + 6) * E))).sum(0))
        add("dD", (p * us).sum(0), (us.abs() * (tp + (rows + 6) * E * p.abs())).sum(0))
        add("dbias", (dd * slope[at]).sum(0),
            out["ddt"][1][at].sum(0) + ((rows + 6) * E * slope[at] * dsize).sum(0))
    return out, last


def scan_inputs(g, rows, n, N, dtype, pad=0, gate=True, full=True):
    s = dict(u=rand(g, rows, n, dtype=dtype, pad=pad), dt=rand(g, rows, n, dtype=dtype, scale=0.7),
             z=rand(g, rows, n, dtype=dtype, pad=pad) if gate else None)
    both = rand(g, rows, 2 * N, dtype=dtype, pad=pad, shift=1 if pad else 0)
    s["Bm"], s["Cm"] = both[:, :N], both[:, N:]
    s["A"] = -torch.exp(torch.randn(n, N, generator=g, device="cuda"))
    s["D"] = torch.randn(n, generator=g, device="cuda") if full else None
    s["bias"] = torch.randn(n, generator=g, device="cuda") * 2 - 3 if full else None
    return s


def pass_on(s):
    return s["u"], s["dt"], s["Bm"], s["Cm"], s["z"]


SCAN_SHAPES = [(1, 1, 1, "one"), (2, 5, 3, "one"), (15, 64, 16, "one"), (17, 65, 16, "one"),
               (130, 70, 16, "ragged"), (700, 33, 16, "ragged"), (400, 130, 8, "ragged"),
               (333, 40, 24, "ragged"), (129, 17, 64, "one"), (80, 20, 33, "ragged"),
               (60, 40, 16, "ones"), (20, 9, 16, "padding"), (640, 257, 16, "one"),
               (200, 100, 15, "ragged")]


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,n,N,kind", SCAN_SHAPES)
@pytest.mark.parametrize("gate,full,pad", [(True, True, 0), (False, False, 3)])
def test_scan(B, dtype, rows, n, N, kind, gate, full, pad):
    g = gen_of(rows + n + N)
    s = scan_inputs(g, rows, n, N, dtype, pad, gate, full)
    dy = rand(g, rows, n, dtype=dtype, pad=pad)
    seq = layout(g, rows, kind)
    runs = [(0, rows, 0)] if seq is None else runs_of(seq)
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for a, r, _ in runs:
        inside[a:a + r] = True
    for t in (s["u"], s["dt"], s["z"], s["Bm"], s["Cm"], dy):
        if t is not None:
            t[~inside] = float("nan")  # of no account
    want, _ = plain_scan(**s, runs=runs, dy=dy)
    op = B.SelectiveScan(s["A"], s["D"], s["bias"])
    y, kept = op.forward(*pass_on(s), seq, keep=True)
    within(y, want["y"], dtype, "y")
    assert torch.equal(op.forward(*pass_on(s), seq), y)
    grads = op.backward(dy, kept)
    assert ("dz" in grads) == gate and ("dD" in grads) == full and ("dbias" in grads) == full
    for k, v in grads.items():
        within(v, want[k], torch.float32 if k in ("dA", "dD", "dbias") else dtype, k)
    for v in [y] + [grads[k] for k in ("du", "ddt", "dB", "dC")]:
        assert (v[~inside] == 0).all()
    again = op.backward(dy, kept)
    assert all(torch.equal(again[k], grads[k]) for k in grads)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("N", [3, 16, 40])
@pytest.mark.parametrize("kind", ["one", "ragged", "ones"])
@pytest.mark.parametrize("same", [True, False])
def test_scan_states(B, dtype, N, kind, same):
    g = gen_of(N)
    rows, n = 450, 37
    s = scan_inputs(g, rows, n, N, dtype)
    seq = layout(g, rows, kind)
    slots = 1 if seq is None else int(seq.max()) + 3
    if kind == "ragged":
        slots -= 5  # the last sequences have no slot: they are padding
    state = torch.randn(slots, n, N, generator=g, device="cuda")
    runs = [(0, rows, 0)] if seq is None else runs_of(seq, slots)
    want, last = plain_scan(**s, runs=runs, state=state)
    op = B.SelectiveScan(s["A"], s["D"], s["bias"])
    before = state.clone()
    out = state if same else torch.full_like(state, 7.0)
    y = op.forward(*pass_on(s), seq, state, out)
    within(y, want["y"], dtype, "y")
    for i in range(slots):
        if i in last:
            check(out[i], last[i][0], last[i][1] + E * last[i][0].abs() + 1e-37, f"state {i}")
        else:
            assert torch.equal(out[i], before[i] if same else torch.full_like(before[i], 7.0))
    if kind == "ones":  # single rows are a step
        again = before.clone()
        y2 = op.step(*pass_on(s), again, seq, again)
        within(y2, want["y"], dtype, "step")
        for i in last:
            check(again[i], last[i][0], last[i][1] + E * last[i][0].abs() + 1e-37, f"step {i}")
        assert torch.equal(op.step(*pass_on(s), before, seq), y2)


def test_scan_in_parts(B):
    """A sequence in parts, one row at a time at its end, is the sequence."""
    g = gen_of(4)
    s = scan_inputs(g, 300, 50, 16, torch.float32)
    op = B.SelectiveScan(s["A"], s["D"], s["bias"])
    want, last = plain_scan(**s, runs=[(0, 300, 0)])
    state = torch.full((1, 50, 16), float("nan"), device="cuda")

    def part(a, e):
        return tuple(t[a:e] for t in pass_on(s))

    out = [op.forward(*part(0, 1), state_out=state)]
    for a, e in ((1, 3), (3, 170), (170, 290)):
        out.append(op.forward(*part(a, e), state=state, state_out=state))
    for t in range(290, 300):
        out.append(op.step(*part(t, t + 1), state=state, state_out=state))
    within(torch.cat(out), want["y"], torch.float32, "y")
    check(state[0], last[0][0], last[0][1] + 1e-37, "state")


def test_scan_states_that_grow(B):
    """An A over 0 whose growth over a chunk is no float: what it meets is 0, or that small."""
    rows, n, N = 1200, 3, 2  # chunks of 32 rows
    g = gen_of(12)
    A = torch.tensor([[1.0, -1.0], [0.97, 0.5], [1.02, -0.1]], device="cuda")
    u, dy = torch.zeros(2, rows, n, device="cuda").unbind()
    dt = torch.full((rows, n), 2.8, device="cuda") + rand(g, rows, n, scale=0.05)
    Bm, Cm = (rand(g, rows, N) for _ in range(2))
    u[31] = 1e-30  # sequence 0 has 70 rows, sequence 1 all others but the last 3
    u[-3:] = 1.0
    dy[:40] = rand(g, 40, n, scale=1e-30)
    dy[80:90] = 1.0
    dy[-3:] = 1.0
    seq = (torch.arange(rows, device="cuda") >= 70).to(torch.int32)
    seq[-3:] = 2
    want, _ = plain_scan(u, dt, Bm, Cm, None, A, None, None, runs_of(seq), dy=dy)
    op = B.SelectiveScan(A)
    y, kept = op.forward(u, dt, Bm, Cm, None, seq, keep=True)
    within(y, want["y"], torch.float32, "y")
    grads = op.backward(dy, kept)
    for k in ("du", "ddt", "dB", "dC", "dA"):
        within(grads[k], want[k], torch.float32, k)


def test_scan_ends_of_softplus(B):
    """Steps from nothing to huge, and decays that leave nothing."""
    x = torch.tensor([-100.0, -60, -20, -1, 0, 1, 20, 88, 1000, 3e4], device="cuda")
    n = len(x)
    u = torch.ones(3, n, device="cuda")
    one = torch.ones(3, 1, device="cuda")
    A = -torch.full((n, 1), 1e-5, device="cuda")
    y = B.SelectiveScan(A).forward(u, x.expand(3, n).contiguous(), one, one)
    want, _ = plain_scan(u, x.expand(3, n), one, one, None, A, None, None, [(0, 3, 0)])
    # under 2^-126 a delta is nothing
    check(y, want["y"][0], want["y"][1] + 4 * E * want["y"][0] + 2.0 ** -125, "y")
    y = B.SelectiveScan(A * 1e7).forward(u, x.expand(3, n).contiguous(), one, one)
    want, _ = plain_scan(u, x.expand(3, n), one, one, None, A * 1e7, None, None, [(0, 3, 0)])
    check(y, want["y"][0], want["y"][1] + 4 * E * want["y"][0] + 2.0 ** -125, "y")


def test_scan_gradient_by_differences(B):
    g = gen_of(8)
    rows, n, N = 90, 6, 4
    s = scan_inputs(g, rows, n, N, torch.float32)
    seq = B.sequences([40, 30, 15], rows)
    runs = runs_of(seq)
    dy = rand(g, rows, n)
    op = B.SelectiveScan(s["A"], s["D"], s["bias"])
    grads = op.backward(dy, op.forward(*pass_on(s), seq, keep=True)[1])
    for name in s:
        v = torch.randn(s[name].shape, generator=g, device="cuda", dtype=torch.float64)
        ends = []
        for sign in (1, -1):
            moved = {**s, name: s[name].double() + sign * 1e-5 * v}
            ends.append(float((plain_scan(**moved, runs=runs)[0]["y"][0] * dy.double()).sum()))
        num = (ends[0] - ends[1]) / 2e-5
        got = grads["d" + name.rstrip("m")].double()
        # third-order terms and 32-bit gradients are far under 1e-5 of the gradient's size
        assert abs(num - float((got * v).sum())) <= 2e-5 * float(got.norm() * v.norm()), name


def test_scan_past_2_31_values(B):
    """u, z, y of more than 2^31 values, the last rows a sequence of their own.  (A call on these rows
    alone cuts them into other chunks: its sums have another order, so 64 bits are the measure.)"""
    rows, n = 540000, 4096
    dtype = torch.bfloat16
    s = {k: torch.zeros(rows, n, dtype=dtype, device="cuda") for k in ("u", "z")}
    tail = scan_inputs(gen_of(1), 64, n, 16, dtype)
    Bm, Cm = (torch.zeros(rows, 16, dtype=dtype, device="cuda") for _ in range(2))
    for name, t in (("u", s["u"]), ("z", s["z"]), ("Bm", Bm), ("Cm", Cm)):
        t[-64:] = tail[name]
    dt = torch.zeros(rows, n, dtype=dtype, device="cuda")
    dt[-64:] = tail["dt"]
    op = B.SelectiveScan(tail["A"], tail["D"], tail["bias"])
    seq = torch.zeros(rows, dtype=torch.int32, device="cuda")
    seq[-64:] = 1
    state = torch.zeros(2, n, 16, device="cuda")
    y = op.forward(s["u"], dt, Bm, Cm, s["z"], seq, state_out=state)
    want, last = plain_scan(**tail, runs=[(0, 64, 0)])
    within(y[-64:], want["y"], dtype, "y")
    check(state[1], last[0][0], last[0][1] + E * last[0][0].abs() + 1e-37, "state")
    assert not y[:-64].any() and not state[0].any()
    del y
    w = rand(gen_of(2), 4, n, dtype=dtype)
    conv = B.CausalConv(w)
    c = conv.forward(s["u"], seq)
    assert torch.equal(c[-64:], conv.forward(tail["u"])) and not c[:-64].any()
    gr = conv.backward(s["u"], s["u"], seq)
    alone = conv.backward(tail["u"], tail["u"])
    assert torch.equal(gr["dx"][-64:], alone["dx"])


# ---------------------------------------------------------------------------------------------
# Streams, graphs, workspaces
# ---------------------------------------------------------------------------------------------
def make(B, seed, rows=700, n=40, N=16, dtype=torch.bfloat16):
    g = gen_of(seed)
    s = scan_inputs(g, rows, n, N, dtype)
    # parameters that a graph reads stay where they are: new values are copied into them
    s.update(x=rand(g, rows, n, dtype=dtype), w=rand(g, 4, n, dtype=dtype),
             dy=rand(g, rows, n, dtype=dtype), seq=layout(g, rows, "ragged"),
             state=torch.randn(40, n, N, generator=g, device="cuda"),
             front=rand(g, 120, n, dtype=dtype).view(40, 3, n).clone())
    return s


def everything(B, s):
    """Each call of both operators; a list of what they return and change."""
    conv, scan = B.CausalConv(s["w"]), B.SelectiveScan(s["A"], s["D"], s["bias"])
    state, front = s["state"].clone(), s["front"].clone()
    out = [conv.forward(s["x"], s["seq"], front, front), *conv.backward(s["dy"], s["x"],
                                                                        s["seq"]).values()]
    out.append(scan.forward(*pass_on(s), s["seq"], state, state))
    y, kept = scan.forward(*pass_on(s), s["seq"], keep=True)
    out += [y, *scan.backward(s["dy"], kept).values()]
    few = tuple(t[:30] for t in pass_on(s))
    out += [conv.step(s["x"][:30], front, None, front), scan.step(*few, state, None, state)]
    return out + [state, front]


def test_mixer_in_a_graph(B):
    """Replays give what eager calls give, with new inputs in the same buffers."""
    a = make(B, 1)
    everything(B, a)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = everything(B, a)
    for seed in (2, 3, 4):
        b = make(B, seed)
        for k, t in b.items():
            a[k].copy_(t)
        graph.replay()
        torch.cuda.synchronize()
        want = everything(B, b)
        torch.cuda.synchronize()
        for i, (x, y) in enumerate(zip(got, want)):
            assert torch.equal(x, y), (seed, i)


def test_mixer_on_two_streams(B):
    a, b = make(B, 1, rows=900), make(B, 2, rows=300, n=70)
    want = everything(B, a), everything(B, b)
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(3):
        for i, (s, stream) in enumerate(zip((a, b), streams)):
            with torch.cuda.stream(stream):
                got[i].append(everything(B, s))
    torch.cuda.synchronize()
    for i in range(2):
        for g in got[i]:
            assert all(torch.equal(x, y) for x, y in zip(g, want[i]))


def test_one_workspace_for_all_rows(lirpa, B):
    """A workspace and a kept buffer for the most rows, full of NaN, serve fewer."""
    n, N, most = 40, 16, 700
    ws = torch.full((max(lirpa.lirpa_scan_workspace_bytes(most, n, N, 1),
                         lirpa.lirpa_conv_workspace_bytes(most, n, 4)) // 4 + 1,), float("nan"),
                    device="cuda").view(torch.uint8)
    kept = torch.full((lirpa.lirpa_scan_kept_bytes(most, n, N) // 4,), float("nan"), device="cuda")
    s = make(B, 5, rows=most)
    op, conv = B.SelectiveScan(s["A"], s["D"], s["bias"]), B.CausalConv(s["w"])
    for rows in (700, 641, 640, 130, 64, 17, 1):
        part = tuple(t[:rows] for t in pass_on(s))
        seq, dy, x = s["seq"][:rows], s["dy"][:rows], s["x"][:rows]
        y, k = op.forward(*part, seq, keep=True)
        want = op.backward(dy, k)
        scan = lirpa.lirpa_scan_inputs(*part, s["A"], s["D"], s["bias"], seq)
        got = torch.empty_like(y)
        lirpa.lirpa_scan_forward(scan, None, None, got, kept, ws, ws.numel())
        assert torch.equal(got, y)
        grads = {name: torch.empty_like(t) for name, t in want.items()}
        order = ("du", "ddt", "dz", "dB", "dC", "dA", "dD", "dbias")
        lirpa.lirpa_scan_backward(scan, dy, kept, *(grads[o] for o in order), ws, ws.numel())
        assert all(torch.equal(grads[o], want[o]) for o in order), rows
        want = conv.backward(dy, x, seq)
        grads = {name: torch.empty_like(t) for name, t in want.items()}
        lirpa.lirpa_conv_backward(dy, x, s["w"], None, "silu", seq, grads["dx"], grads["dw"], None,
                                  ws, ws.numel())
        assert all(torch.equal(grads[o], want[o]) for o in grads), rows


def test_no_rows(B):
    A = torch.randn(12, 5, device="cuda")
    op = B.SelectiveScan(A, A[:, 0].contiguous(), A[:, 1].contiguous())
    x, b = torch.empty(0, 12, device="cuda"), torch.empty(0, 5, device="cuda")
    y, kept = op.forward(x, x, b, b, x, keep=True)
    grads = op.backward(x, kept)
    assert y.shape == (0, 12)
    assert all((grads[k] == 0).all() for k in ("dA", "dD", "dbias"))
    conv = B.CausalConv(torch.randn(4, 12, device="cuda"), torch.randn(12, device="cuda"))
    assert conv.forward(x).shape == (0, 12)
    g = conv.backward(x, x)
    assert (g["dw"] == 0).all() and (g["dbias"] == 0).all()


def test_binding_checks(B):
    s = make(B, 3, rows=50)
    op, conv = B.SelectiveScan(s["A"], s["D"], s["bias"]), B.CausalConv(s["w"])
    with pytest.raises(ValueError, match="state must be"):
        op.forward(*pass_on(s), state=s["state"][:, :, :8])
    with pytest.raises(TypeError, match="state"):
        op.forward(*pass_on(s), state=s["state"].half())
    with pytest.raises(ValueError, match="slots"):
        op.forward(*pass_on(s), state=s["state"], state_out=s["state"][:3].clone())
    with pytest.raises(ValueError, match="exclude"):
        op.forward(*pass_on(s), state=s["state"], keep=True)
    with pytest.raises(TypeError, match="seq"):
        op.forward(*pass_on(s), s["seq"].long())
    with pytest.raises(ValueError, match="seq"):
        conv.forward(s["x"], s["seq"][:30])
    with pytest.raises(ValueError, match="state must be"):
        conv.forward(s["x"], state=s["front"][:, :2])
    with pytest.raises(TypeError, match="dt"):
        op.forward(s["u"], s["dt"].float(), s["Bm"], s["Cm"])
    with pytest.raises(ValueError, match="A must have"):
        B.SelectiveScan(s["A"][:30].contiguous()).forward(*pass_on(s))
    with pytest.warns(UserWarning, match="autograd"):
        conv.forward(s["x"].clone().requires_grad_())
    with pytest.warns(UserWarning, match="autograd"):
        op.forward(s["u"].clone().requires_grad_(), *pass_on(s)[1:])


# ---------------------------------------------------------------------------------------------
# Gradients where the last sequences have no slot
# ---------------------------------------------------------------------------------------------
def slotless(g, rows, *tensors):
    """(seq, slots, runs, rows of sequences with a slot): the last sequences have none, and hold NaN
    in the given tensors."""
    seq = layout(g, rows, "ragged")
    slots = int(seq.max()) - 2
    runs = runs_of(seq, slots)
    assert 0 < len(runs) < len(runs_of(seq))
    inside = torch.zeros(rows, dtype=torch.bool, device="cuda")
    for a, r, _ in runs:
        inside[a:a + r] = True
    for t in tensors:
        t[~inside] = float("nan")
    return seq, slots, runs, inside


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,n,N", [(450, 37, 16), (450, 70, 5), (130, 20, 40), (1500, 33, 16)])
def test_scan_gradient_of_rows_without_a_slot(B, lirpa, dtype, rows, n, N):
    """What was padding in the forward pass is so in the backward pass, whatever came between."""
    g = gen_of(rows + N)
    s = scan_inputs(g, rows, n, N, dtype)
    dy = rand(g, rows, n, dtype=dtype)
    seq, slots, runs, inside = slotless(g, rows, dy, *pass_on(s))
    want, last = plain_scan(**s, runs=runs, dy=dy)
    op = B.SelectiveScan(s["A"], s["D"], s["bias"])
    out = torch.zeros(slots, n, N, device="cuda")
    y, kept = op.forward(*pass_on(s), seq, state_out=out, keep=True)
    within(y, want["y"], dtype, "y")
    for _, _, i in runs:
        check(out[i], last[i][0], last[i][1] + E * last[i][0].abs() + 1e-37, f"state {i}")
    assert kept.slots == slots
    grads = op.backward(dy, kept)
    for k, v in grads.items():
        within(v, want[k], torch.float32 if k in ("dA", "dD", "dbias") else dtype, k)
    for k in ("du", "ddt", "dz", "dB", "dC"):
        assert (grads[k][~inside] == 0).all(), k

    # the library's calls on one lirpa_scan: a call without kept leaves the gradient's slots alone
    scan = lirpa.lirpa_scan_inputs(*pass_on(s), s["A"], s["D"], s["bias"], seq)
    size = (rows, n, N)
    states = torch.empty(lirpa.lirpa_scan_kept_bytes(*size), dtype=torch.uint8, device="cuda")
    need = max(lirpa.lirpa_scan_workspace_bytes(*size, back) for back in (0, 1))
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    y2 = torch.empty_like(y)
    lirpa.lirpa_scan_forward(scan, None, out, y2, states, ws, need)
    assert torch.equal(y2, y)
    many = torch.zeros(slots + 9, n, N, device="cuda")
    lirpa.lirpa_scan_forward(scan, None, many, torch.empty_like(y), None, ws, need)
    lirpa.lirpa_scan_step(scan, many, None, torch.empty_like(y))
    assert scan.slots == lirpa.ANY_SLOT
    order = ("du", "ddt", "dz", "dB", "dC", "dA", "dD", "dbias")
    for more in ({}, {"slots": slots}):
        again = {k: torch.empty_like(grads[k]) for k in order}
        lirpa.lirpa_scan_backward(scan, dy, states, *again.values(), ws, need, **more)
        assert all(torch.equal(again[k], grads[k]) for k in order)

    # without states the scan's own slots hold
    scan = lirpa.lirpa_scan_inputs(*pass_on(s), s["A"], s["D"], s["bias"], seq, slots)
    lirpa.lirpa_scan_forward(scan, None, None, y2.fill_(7.0), states, ws, need)
    assert torch.equal(y2, y)
    with pytest.raises(ValueError, match="slots"):
        lirpa.lirpa_scan_backward(scan, dy, states, *again.values(), ws, need, slots=1 << 31)


@pytest.mark.parametrize("dtype", TYPES, ids=ids)
@pytest.mark.parametrize("rows,n,taps", [(450, 37, 4), (130, 20, 8), (1500, 130, 3)])
def test_conv_gradient_of_rows_without_a_slot(B, dtype, rows, n, taps):
    g = gen_of(rows + taps)
    x, dy = (rand(g, rows, n, dtype=dtype) for _ in range(2))
    w, b = rand(g, taps, n, dtype=dtype), rand(g, 1, n, dtype=dtype)[0]
    seq, slots, runs, inside = slotless(g, rows, x, dy)
    op = B.CausalConv(w, b)
    want, _ = plain_conv(x, w, b, "silu", runs, dy=dy)
    out = torch.zeros(slots, taps - 1, n, dtype=dtype, device="cuda")
    within(op.forward(x, seq, state_out=out), want["y"], dtype, "y")
    grads = op.backward(dy, x, seq, slots)
    for k, v in grads.items():
        within(v, want[k], dtype, k)
    assert (grads["dx"][~inside] == 0).all()
    for bad in (0, -1, 1 << 31, (1 << 32) + 3):
        with pytest.raises(ValueError, match="slots"):
            op.backward(dy, x, seq, bad)


def test_scan_gradient_past_2_31_values(B):
    """Inputs, gradients, kept states and parts of dB and dC of more than 2^31 values each, the last
    rows a sequence of their own, the others zeros."""
    rows, n, N = 540000, 4096, 32
    dtype = torch.bfloat16
    g = gen_of(3)
    tail = scan_inputs(g, 64, n, N, dtype)
    dy_tail = rand(g, 64, n, dtype=dtype)
    whole = {k: torch.zeros(rows, t.shape[1], dtype=dtype, device="cuda")
             for k, t in {**tail, "dy": dy_tail}.items() if k in ("u", "dt", "z", "Bm", "Cm", "dy")}
    for k, t in whole.items():
        t[-64:] = dy_tail if k == "dy" else tail[k]
    seq = torch.zeros(rows, dtype=torch.int32, device="cuda")
    seq[-64:] = 1
    op = B.SelectiveScan(tail["A"], tail["D"], tail["bias"])
    y, kept = op.forward(*pass_on(whole), seq, keep=True)
    assert kept.states.numel() > 1 << 33 and not y[:-64].any()
    del y
    grads = op.backward(whole["dy"], kept)
    want, _ = plain_scan(**tail, runs=[(0, 64, 0)], dy=dy_tail)
    for k, v in grads.items():
        if k in ("dA", "dD", "dbias"):
            within(v, want[k], torch.float32, k)
        else:
            within(v[-64:], want[k], dtype, k)
            assert not v[:-64].any(), k
