"""A language model's operators around its feed-forward blocks, as calls to time and compare.

The operators are those of ``paper_2011_13824_amd.blocks``:

* ``embed``        rows of a table by token, scaled; a token outside the table is padding, a row of 0;
* ``embed_back``   the table's gradient: the rows of each token summed, with ``add`` onto the rest
                   of that gradient (the table is the last layer's weight too);
* ``logprob``      log probabilities of given tokens, log of the sum, entropy and the ``top`` most
                   likely tokens of every row of logits;
* ``logprob_back`` the gradient of the logits, from those of the log probabilities and entropies;
* ``conv``         short causal convolution of every column, with silu, over sequences that lie
                   behind each other, with the last inputs of a sequence as its state;
* ``conv_train``   both passes of it;
* ``scan``         the selective state space scan h_t = exp(delta A) h_{t-1} + delta u B,
                   y = (C h + D u) silu(z), delta = softplus(dt + bias), with states in and out;
* ``scan_train``   both passes of it, from states of 0;
* ``step``         one token of every sequence: a convolution's and a scan's, states in and out.

The plain forms compute in 32 bits with elementary operations and round once at the end.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def listed():
    return [
        # the tokens of prompts on their way into a model
        dict(name="embed_prompt", op="embed", type="bf16", rows=8192, n=4096, vocab=128000, pad=0),
        # the table's gradient in a training step: most of it is rows that no token named
        dict(name="embed_back", op="embed_back", type="bf16", rows=16384, n=4096, vocab=128000,
             add=False, pad=0),
        # a 32-bit model of odd width whose table is its last layer's weight too
        dict(name="embed_back_tied", op="embed_back", type="f32", rows=2999, n=1001, vocab=32003,
             add=True, pad=3),
        # an answer's next token: its log probability and the alternatives shown with it
        dict(name="logprob_token", op="logprob", type="bf16", rows=1, n=128000, top=20, scale=1.0,
             pad=0),
        # new tokens of many sequences, a vocabulary of odd size, sampled at a temperature
        dict(name="logprob_few", op="logprob", type="f32", rows=61, n=50001, top=5, scale=1.25,
             pad=7),
        # the loss of a training step
        dict(name="logprob_train", op="logprob", type="bf16", rows=4096, n=128000, top=0,
             scale=1.0, pad=0),
        # its gradient, with that of an entropy term
        dict(name="logprob_back", op="logprob_back", type="bf16", rows=4096, n=128000, scale=1.0,
             pad=0),
        # a long prompt, read in parts: the convolution starts from the last part's inputs
        dict(name="conv_prompt", op="conv", type="bf16", rows=8192, n=4096, taps=4, seqs=1, pad=0),
        # training on a ragged batch whose rows are half of a wider projection
        dict(name="conv_train", op="conv_train", type="f16", rows=4099, n=1001, taps=4, seqs=7,
             pad=1001),
        # the scan of that long prompt
        dict(name="scan_prompt", op="scan", type="bf16", rows=8192, n=4096, states=16, seqs=1,
             pad=0),
        # training on documents of any length behind each other
        dict(name="scan_train", op="scan_train", type="bf16", rows=8192, n=4096, states=16, seqs=5,
             pad=0),
        # serving: one new token of each of many sequences
        dict(name="step", op="step", type="bf16", rows=48, n=4096, states=16, taps=4, pad=0),
    ]


def _log(rng, lo, hi, step=1):
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    return min(hi, max(lo, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["embed", "embed_back", "logprob", "logprob_back", "conv", "conv_train", "scan",
                     "scan_train", "step"])
    case = dict(op=op, type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                pad=rng.choice([0, 0, 8, 5]))
    step = rng.choice([1, 8, 64, 64])  # odd widths, those of whole 16-byte pieces, usual ones
    half = 2 if case["type"] == "f32" else 1
    if op in ("embed", "embed_back"):
        n = _log(rng, 64, 4096, step)
        vocab = min(_log(rng, 1000, 128000), 128000 * 4096 // (n * half))
        rows = min(_log(rng, 1, 16384), 16384 * 4096 // (n * half))
        case.update(rows=rows, n=n, vocab=vocab)
        if op == "embed_back":
            case["add"] = rng.random() < 0.4
        return case
    if op in ("logprob", "logprob_back"):
        n = _log(rng, 1000, 128000, step)
        rows = min(_log(rng, 1, 4096), 4096 * 128000 // (n * half))
        case.update(rows=rows, n=n, scale=rng.choice([1.0, 1.0, 0.7, 1.25]))
        if op == "logprob":
            case["top"] = rng.choice([0, 1, 5, 20]) if rows <= 256 else 0
        return case
    n = _log(rng, 64, 4096, step)
    if op == "step":
        case.update(rows=_log(rng, 1, 256), n=n, states=rng.choice([8, 16, 16, 24]),
                    taps=rng.choice([2, 3, 4]))
        return case
    rows = _log(rng, 1, 8192)
    if op in ("scan", "scan_train"):
        case.update(rows=rows, n=n, states=rng.choice([8, 16, 16, 16, 24]))
        if case["states"] > 16 or case["type"] == "f32":
            case["rows"] = min(rows, 8192 * 4096 // (2 * n))
    else:
        case.update(rows=min(rows, 8192 * 4096 // (n * half)), n=n, taps=rng.choice([2, 3, 4]))
    case["seqs"] = min(case["rows"], rng.choice([1, 2, 5, 16, 40]))
    return case


# ---------------------------------------------------------------------------------------------
# inputs


def _rows(gen, rows, n, pad, kind, spread=1.0):
    """A [rows, n] view into rows of n + pad values."""
    x = torch.randn(rows, n + pad, generator=gen, device="cuda", dtype=torch.float32)
    return (x * spread).to(TYPES[kind])[:, :n]


def _tokens(gen, rows, vocab):
    """Tokens as text has them, the k-th frequent one about 1 / k as often as the first; their
    numbers are in no order.  One row in 64 is padding."""
    u = torch.rand(rows, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(vocab + 1)).long() - 1).clamp(0, vocab - 1)
    tokens = torch.randperm(vocab, generator=gen, device="cuda")[rank]
    tokens[torch.rand(rows, generator=gen, device="cuda") < 1 / 64] = -1
    return tokens


def _sequences(gen, rows, seqs):
    """[(first row, rows)] of `seqs` sequences of any length; a ragged batch ends with a few rows
    of padding."""
    spare = rows // 100 if seqs > 1 else 0
    cuts = torch.randperm(rows - spare - 1, generator=gen, device="cuda")[:seqs - 1] + 1 \
        if seqs > 1 and rows - spare > seqs else torch.arange(1, seqs, device="cuda")
    ends = sorted(cuts.tolist()) + [rows - spare]
    return [(a, b - a) for a, b in zip([0] + ends[:-1], ends)]


def _scan_inputs(s, gen, rows, n, pad, kind):
    states = s["states"]
    s["u"] = _rows(gen, rows, n, pad, kind)
    s["dt"] = _rows(gen, rows, n, 0, kind, 0.5)
    s["z"] = _rows(gen, rows, n, pad, kind)
    both = _rows(gen, rows, 2 * states, pad, kind)  # B and C come out of one projection
    s["B"], s["C"] = both[:, :states], both[:, states:]
    s["A"] = -(torch.arange(1, states + 1, device="cuda")
               * torch.exp(0.1 * torch.randn(n, states, generator=gen, device="cuda")))
    s["D"] = 1 + 0.1 * torch.randn(n, generator=gen, device="cuda")
    # steps of 0.001 to 0.1 where dt is 0
    step = torch.exp(torch.rand(n, generator=gen, device="cuda") * math.log(100.0)) * 0.001
    s["bias"] = step + torch.log(-torch.expm1(-step))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed))
    op, kind, rows, n, pad = (case[k] for k in ("op", "type", "rows", "n", "pad"))
    s = dict(case)
    if op in ("embed", "embed_back"):
        s["tokens"] = _tokens(gen, rows, case["vocab"])
        s["factor"] = n ** 0.5
        if op == "embed":
            s["table"] = _rows(gen, case["vocab"], n, pad, kind, n ** -0.5)
        else:
            s["dout"] = _rows(gen, rows, n, pad, kind)
            s["table"] = _rows(gen, case["vocab"], n, 0, kind, n ** -0.5)
            if case["add"]:
                s["before"] = _rows(gen, case["vocab"], n, 0, kind)
    elif op in ("logprob", "logprob_back"):
        s["logits"] = _rows(gen, rows, n, pad, kind, 2.5)
        s["tokens"] = torch.randint(0, n, (rows,), generator=gen, device="cuda")
        # a model that has learned something: most given tokens are among the likely ones
        s["logits"][torch.arange(rows, device="cuda"), s["tokens"]] += 8
        if rows > 64:
            s["tokens"][torch.rand(rows, generator=gen, device="cuda") < 1 / 64] = -1
        if op == "logprob_back":
            s["dlogp"] = -torch.rand(rows, generator=gen, device="cuda") / rows
            s["dentropy"] = -0.01 * torch.rand(rows, generator=gen, device="cuda") / rows
            s["lse"], s["entropy"] = _moments(s["logits"], case["scale"])[1:]
    else:
        taps = case.get("taps", 0)
        if op == "step":
            s["seqs"] = rows
            s["runs"] = [(i, 1) for i in range(rows)]
        else:
            s["runs"] = _sequences(gen, rows, case["seqs"])
        # the slots of the sequences in a cache that has a few more
        s["slots"] = case.get("seqs", rows) + 3
        order = torch.randperm(s["slots"], generator=gen, device="cuda")[:len(s["runs"])]
        s["order"] = order.tolist()
        if op == "step":
            s["seq"] = order.to(torch.int32)
        elif len(s["runs"]) > 1 or op in ("conv", "scan"):
            lens = torch.tensor([r for _, r in s["runs"]], device="cuda")
            seq = torch.full((rows,), -1, dtype=torch.int32, device="cuda")
            seq[:int(lens.sum())] = torch.repeat_interleave(order.to(torch.int32), lens)
            s["seq"] = seq
        else:
            s["seq"], s["order"] = None, [0]
        if taps:
            s["x"] = _rows(gen, rows, n, pad, kind)
            s["w"] = _rows(gen, taps, n, 0, kind, taps ** -0.5)
            s["wbias"] = _rows(gen, 1, n, 0, kind, 0.1)[0]
            if op != "conv_train":
                s["inputs"] = _rows(gen, s["slots"] * (taps - 1), n, 0, kind).view(
                    s["slots"], taps - 1, n)
        if case.get("states"):
            _scan_inputs(s, gen, rows, n, pad, kind)
            if op != "scan_train":
                s["h0"] = torch.randn(s["slots"], n, case["states"], generator=gen, device="cuda")
        if op in ("conv_train", "scan_train"):
            s["dy"] = _rows(gen, rows, n, 0, kind)
        # where the states go: a buffer of its own, so that a pass can be repeated
        s["inputs_out"] = s["inputs"].clone() if "inputs" in s else None
        s["h_out"] = s["h0"].clone() if "h0" in s else None
    if own:
        from paper_2011_13824_amd import blocks
        if op in ("embed", "embed_back"):
            s["op_embed"] = blocks.Embedding(s["table"], s["factor"])
        elif op in ("logprob", "logprob_back"):
            s["op_logprob"] = blocks.LogProbs(case["scale"], case.get("top", 0))
        if case.get("taps"):
            s["op_conv"] = blocks.CausalConv(s["w"], s["wbias"], "silu")
        if case.get("states"):
            s["op_scan"] = blocks.SelectiveScan(s["A"], s["D"], s["bias"])
    return s


# ---------------------------------------------------------------------------------------------
# plain forms


def _embed(s):
    t = s["tokens"]
    out = s["table"][t.clamp(min=0)].float() * s["factor"]
    return {"out": (out * (t >= 0)[:, None]).to(s["table"].dtype)}


def _embed_back(s):
    t = s["tokens"]
    total = torch.zeros(s["vocab"] + 1, s["n"], device="cuda")
    total.index_add_(0, torch.where(t >= 0, t, s["vocab"]), s["dout"].float())
    total = total[:-1] * s["factor"]
    if s["add"]:
        total = total + s["before"].float()
    return {"dtable": total.to(s["dout"].dtype)}


def _moments(logits, scale):
    """(scaled logits, log of the sum of their exponentials, entropy)"""
    x = logits.float() * scale
    top = x.amax(1, keepdim=True)
    d = x - top
    e = torch.exp(d)
    total = e.sum(1)
    log = torch.log(total)
    return x, top[:, 0] + log, log - (e * d).sum(1) / total


def _logprob(s):
    x, lse, entropy = _moments(s["logits"], s["scale"])
    t = s["tokens"]
    at = x.gather(1, t.clamp(min=0)[:, None])[:, 0]
    out = {"logp": torch.where(t >= 0, at - lse, 0.0), "lse": lse, "entropy": entropy}
    if s["top"]:
        left, columns = s["logits"].float(), torch.arange(s["n"], device="cuda")
        values, indices = [], []
        for _ in range(s["top"]):
            best = left.amax(1, keepdim=True)
            i = torch.where(left == best, columns, s["n"]).amin(1, keepdim=True)
            left = left.scatter(1, i, -math.inf)
            values.append(best[:, 0] * s["scale"] - lse)
            indices.append(i[:, 0])
        out["top_logp"], out["top_tokens"] = torch.stack(values, 1), torch.stack(indices, 1)
    return out


def _logprob_back(s):
    t, scale = s["tokens"], s["scale"]
    log_p = s["logits"].float() * scale - s["lse"][:, None]
    p = torch.exp(log_p)
    g = torch.where(t >= 0, s["dlogp"], 0.0)[:, None]
    d = -p * (g + s["dentropy"][:, None] * (log_p + s["entropy"][:, None]))
    d.scatter_add_(1, t.clamp(min=0)[:, None], g)
    return {"dlogits": (d * scale).to(s["logits"].dtype)}


def _pre(s, states):
    """The convolution's sums before the activation, every sequence behind its state, and the
    inputs with those in front."""
    x, w, taps = s["x"].float(), s["w"].float(), s["taps"]
    pre = torch.zeros_like(x)
    padded = []
    for (a, r), slot in zip(s["runs"], s["order"]):
        front = states[slot].float() if states is not None else x.new_zeros(taps - 1, s["n"])
        p = torch.cat([front, x[a:a + r]])
        pre[a:a + r] = s["wbias"].float()
        for k in range(taps):
            pre[a:a + r] += w[k] * p[k:k + r]
        padded.append(p)
    return pre, padded


def _silu(x):
    """(x / (1 + exp(-x)), its slope)"""
    p = torch.sigmoid(x)
    return x * p, p * (1 + x * (1 - p))


def _inside(s, rows):
    """1 for the rows of sequences, 0 behind the last one."""
    last = s["runs"][-1]
    return (torch.arange(rows, device="cuda") < last[0] + last[1]).float()[:, None]


def _conv(s):
    pre, padded = _pre(s, s["inputs"])
    out = s["inputs_out"].clone()
    for p, slot in zip(padded, s["order"]):
        out[slot] = p[p.shape[0] - (s["taps"] - 1):].to(out.dtype)
    y = _silu(pre)[0] * _inside(s, s["rows"])
    return {"y": y.to(s["x"].dtype), "inputs": out}


def _conv_train(s):
    kind = s["x"].dtype
    pre, padded = _pre(s, None)
    y, slope = _silu(pre)
    inside = _inside(s, s["rows"])
    d = s["dy"].float() * slope * inside
    w, taps = s["w"].float(), s["taps"]
    dx, dw = torch.zeros_like(d), torch.zeros_like(w)
    for (a, r), p in zip(s["runs"], padded):
        behind = torch.cat([d[a:a + r], d.new_zeros(taps - 1, s["n"])])
        for k in range(taps):
            dx[a:a + r] += w[k] * behind[taps - 1 - k:taps - 1 - k + r]
            dw[k] += (d[a:a + r] * p[k:k + r]).sum(0)
    return {"y": (y * inside).to(kind), "dx": dx.to(kind), "dw": dw.to(kind),
            "dbias": d.sum(0).to(kind)}


def _scan(s, train=False):
    kind = s["u"].dtype
    u, B, C, z = (s[k].float() for k in ("u", "B", "C", "z"))
    x = s["dt"].float() + s["bias"]
    delta = x.clamp(min=0) + torch.log1p(torch.exp(-x.abs()))
    a = torch.exp(delta[:, :, None] * s["A"])
    b = (delta * u)[:, :, None] * B[:, None, :]
    h = torch.zeros_like(a)
    out = s["h_out"].clone() if not train else None
    for (first, r), slot in zip(s["runs"], s["order"]):
        last = s["h0"][slot] if not train else torch.zeros_like(a[0])
        for t in range(first, first + r):
            torch.addcmul(b[t], a[t], last, out=h[t])
            last = h[t]
        if not train:
            out[slot] = last
    y = torch.einsum("tdn,tn->td", h, C) + s["D"] * u
    inside = _inside(s, s["rows"])
    gate, slope = _silu(z)
    result = {"y": (y * gate * inside).to(kind)}
    if not train:
        return {**result, "h": out}
    dy = s["dy"].float() * inside
    dz = dy * y * slope
    p = dy * gate
    dC = torch.einsum("td,tdn->tn", p, h)
    before = torch.zeros_like(h)  # h of the row before, 0 at a sequence's first
    before[1:] = h[:-1]
    for first, _ in s["runs"]:
        before[first] = 0
    g = p[:, :, None] * C[:, None, :]
    for first, r in s["runs"]:
        for t in range(first + r - 2, first - 1, -1):
            g[t].addcmul_(a[t + 1], g[t + 1])
    gB = torch.einsum("tdn,tn->td", g, B)
    dB = torch.einsum("tdn,td->tn", g, delta * u)
    e = g.mul_(a).mul_(before)
    ddelta = torch.einsum("tdn,dn->td", e, s["A"]) + u * gB
    ddt = ddelta * torch.sigmoid(x)
    result.update(du=(delta * gB + s["D"] * p).to(kind), ddt=ddt.to(kind), dz=dz.to(kind),
                  dB=dB.to(kind), dC=dC.to(kind), dA=torch.einsum("tdn,td->dn", e, delta),
                  dD=(p * u).sum(0), dbias=ddt.sum(0))
    return result


def _step(s):
    first = _conv(s)
    return {**_scan(s), "x": first["y"], "inputs": first["inputs"]}


def _plain(s):
    return {"embed": _embed, "embed_back": _embed_back, "logprob": _logprob,
            "logprob_back": _logprob_back, "conv": _conv, "conv_train": _conv_train, "scan": _scan,
            "scan_train": lambda s: _scan(s, train=True), "step": _step}[s["op"]](s)


# ---------------------------------------------------------------------------------------------
# the library's calls


def _library(s):
    op = s["op"]
    if op == "embed":
        return {"out": s["op_embed"].forward(s["tokens"])}
    if op == "embed_back":
        return {"dtable": s["op_embed"].backward(s["tokens"], s["dout"], base=s.get("before"))}
    if op == "logprob":
        r = s["op_logprob"].forward(s["logits"], s["tokens"])
        out = {"logp": r.logp, "lse": r.lse, "entropy": r.entropy}
        if s["top"]:
            out["top_logp"], out["top_tokens"] = r.top_logp, r.top_tokens
        return out
    if op == "logprob_back":
        return {"dlogits": s["op_logprob"].backward(s["logits"], s["tokens"], s["lse"],
                                                    s["entropy"], s["dlogp"], s["dentropy"])}
    if op == "conv":
        y = s["op_conv"].forward(s["x"], s["seq"], s["inputs"], s["inputs_out"])
        return {"y": y, "inputs": s["inputs_out"]}
    if op == "conv_train":
        y = s["op_conv"].forward(s["x"], s["seq"])
        return {"y": y, **s["op_conv"].backward(s["dy"], s["x"], s["seq"])}
    if op == "scan":
        y = s["op_scan"].forward(s["u"], s["dt"], s["B"], s["C"], s["z"], s["seq"], s["h0"],
                                 s["h_out"])
        return {"y": y, "h": s["h_out"]}
    if op == "scan_train":
        y, kept = s["op_scan"].forward(s["u"], s["dt"], s["B"], s["C"], s["z"], s["seq"], keep=True)
        return {"y": y, **s["op_scan"].backward(s["dy"], kept)}
    x = s["op_conv"].step(s["x"], s["inputs"], s["seq"], s["inputs_out"])
    y = s["op_scan"].step(s["u"], s["dt"], s["B"], s["C"], s["z"], s["h0"], s["seq"], s["h_out"])
    return {"y": y, "h": s["h_out"], "x": x, "inputs": s["inputs_out"]}


def run(state):
    return _library(state) if own else _plain(state)


def work(case):
    op, rows, n = case["op"], case["rows"], case["n"]
    size = 4 if case["type"] == "f32" else 2
    whole = rows * n * size
    if op == "embed":
        return {"bytes": 8 * rows + 2 * whole, "flops": rows * n}
    if op == "embed_back":
        table = (2 if case["add"] else 1) * case["vocab"] * n * size
        return {"bytes": 8 * rows + whole + table, "flops": rows * n}
    if op == "logprob":
        return {"bytes": whole + rows * (8 + 12 + 12 * case["top"]), "flops": 7 * rows * n}
    if op == "logprob_back":
        return {"bytes": 2 * whole + rows * 24, "flops": 7 * rows * n}
    taps = case.get("taps", 0)
    front = 2 * case.get("seqs", rows) * max(taps - 1, 0) * n * size  # a sequence's last inputs
    if op == "conv":
        return {"bytes": 2 * whole + front, "flops": (2 * taps + 4) * rows * n}
    if op == "conv_train":
        return {"bytes": 5 * whole, "flops": (8 * taps + 14) * rows * n}
    states = case["states"]
    both = 2 * rows * states * size
    h = 2 * case.get("seqs", rows) * n * states * 4  # states read and written
    if op == "scan":
        return {"bytes": 4 * whole + both + h, "flops": (7 * states + 12) * rows * n}
    if op == "scan_train":
        return {"bytes": 11 * whole + 3 * both, "flops": (30 * states + 40) * rows * n}
    return {"bytes": 6 * whole + both + h + front, "flops": (7 * states + 2 * taps + 16) * rows * n}


# ---------------------------------------------------------------------------------------------
# the definitions in 64 bits


def _exact_conv(d, s, x, states):
    """Rows of the definition: activation of bias + sum_k w_k x_{t - taps + 1 + k}."""
    rows = []
    taps = s["taps"]
    for (a, r), slot in zip(s["runs"], s["order"]):
        seq = x[a:a + r]
        if states is not None:
            seq = torch.cat([states[slot], seq])
        else:
            seq = torch.nn.functional.pad(seq, (0, 0, taps - 1, 0))
        windows = seq.unfold(0, taps, 1)  # [rows, columns, taps]
        pre = torch.einsum("tdk,kd->td", windows, d["w"]) + d["wbias"]
        rows.append(pre / (1 + torch.exp(-pre)))
    behind = s["rows"] - sum(r for _, r in s["runs"])
    return torch.cat(rows + [x.new_zeros(behind, s["n"])])


def _exact_front(d, s):
    out = d["inputs_out"].clone()
    for (a, r), slot in zip(s["runs"], s["order"]):
        for k in range(s["taps"] - 1):  # input number t of the sequence, its state's in front
            t = r - (s["taps"] - 1) + k
            out[slot, k] = d["x"][a + t] if t >= 0 else d["inputs"][slot, t + s["taps"] - 1]
    return out


def _exact_scan(d, s, u, states):
    """(y, last states): a walk over the rows of each sequence."""
    ys, last = [], []
    for (a, r), slot in zip(s["runs"], s["order"]):
        step = torch.logaddexp(d["dt"][a:a + r] + d["bias"], torch.zeros_like(d["bias"]))
        h = states[slot] if states is not None else torch.zeros_like(d["A"])
        for delta, v, B, C in zip(step, u[a:a + r], d["B"][a:a + r], d["C"][a:a + r]):
            h = h * torch.exp(delta.unsqueeze(1) * d["A"]) + torch.outer(delta * v, B)
            ys.append(h.mv(C))
        last.append(h)
    y = torch.stack(ys)
    z = d["z"][:len(ys)]
    y = (y + u[:len(ys)] * d["D"]) * z / (1 + torch.exp(-z))
    behind = s["rows"] - len(ys)
    return torch.cat([y, y.new_zeros(behind, s["n"])]), last


def _exact_states(d, s, last):
    out = d["h_out"].clone()
    for h, slot in zip(last, s["order"]):
        out[slot] = h
    return out


def exact(case, seed):
    global own
    kept_own, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = kept_own
    d = {k: v.double() for k, v in s.items()
         if isinstance(v, torch.Tensor) and v.is_floating_point()}
    op, rows, n, t = case["op"], case["rows"], case["n"], s.get("tokens")
    if op == "embed":
        out = torch.zeros(rows, n, dtype=torch.float64, device="cuda")
        named = t.ge(0).nonzero()[:, 0]
        out[named] = d["table"].index_select(0, t[named]) * s["factor"]
        return {"out": out}
    if op == "embed_back":
        total = torch.zeros(case["vocab"], n, dtype=torch.float64, device="cuda")
        named = t.ge(0).nonzero()[:, 0]
        total.index_put_((t[named],), s["factor"] * d["dout"][named], accumulate=True)
        return {"dtable": total + d["before"] if case["add"] else total}
    if op in ("logprob", "logprob_back"):
        log_p = torch.log_softmax(d.pop("logits") * case["scale"], 1)
        p = torch.exp(log_p)
        entropy = -torch.einsum("ij,ij->i", p, log_p)
        if op == "logprob":
            out = {"logp": torch.zeros(rows, dtype=torch.float64, device="cuda"),
                   "lse": torch.logsumexp(s["logits"].double() * case["scale"], 1),
                   "entropy": entropy}
            for i in t.ge(0).nonzero()[:, 0].tolist():
                out["logp"][i] = log_p[i, t[i]]
            if case["top"]:
                order = torch.argsort(-s["logits"].double(), dim=1, stable=True)[:, :case["top"]]
                out["top_tokens"], out["top_logp"] = order, torch.gather(log_p, 1, order)
            return out
        # the gradient at the entropies and sums that the call is given, in 32 bits
        log_p = s["logits"].double() * case["scale"] - d["lse"].unsqueeze(1)
        p = torch.exp(log_p)
        g = d["dlogp"] * (t >= 0)
        slope = log_p.add_(d["entropy"].unsqueeze(1)).mul_(d["dentropy"].unsqueeze(1))
        grad = slope.add_(g.unsqueeze(1)).mul_(p).neg_()
        named = t.ge(0).nonzero()[:, 0]
        grad[named, t[named]] += g[named]
        return {"dlogits": grad.mul_(case["scale"])}
    if op == "conv":
        return {"y": _exact_conv(d, s, d["x"], d["inputs"]), "inputs": _exact_front(d, s)}
    if op == "scan":
        y, last = _exact_scan(d, s, d["u"], d["h0"])
        return {"y": y, "h": _exact_states(d, s, last)}
    if op == "step":
        y, last = _exact_scan(d, s, d["u"], d["h0"])
        return {"y": y, "h": _exact_states(d, s, last),
                "x": _exact_conv(d, s, d["x"], d["inputs"]), "inputs": _exact_front(d, s)}
    # the training steps: gradients by autograd from the definition, columns in parts
    if op == "conv_train":
        for k in ("x", "w", "wbias"):
            d[k].requires_grad_()
        y = _exact_conv(d, s, d["x"], None)
        dx, dw, db = torch.autograd.grad(y, (d["x"], d["w"], d["wbias"]), d["dy"])
        return {"y": y.detach(), "dx": dx, "dw": dw, "dbias": db}
    parts = []
    width = max(1, (2 << 30) // (rows * case["states"]))
    for c in range(0, n, width):
        at = slice(c, min(n, c + width))
        q = {k: d[k][:, at] for k in ("u", "dt", "z")}
        q.update({k: d[k][at] for k in ("A", "D", "bias")}, B=d["B"], C=d["C"])
        q = {k: v.detach().clone().requires_grad_() for k, v in q.items()}
        y, _ = _exact_scan(q, {**s, "n": at.stop - c}, q["u"], None)
        names = ("u", "dt", "z", "A", "D", "bias", "B", "C")
        grads = torch.autograd.grad(y, [q[k] for k in names], d["dy"][:, at])
        parts.append({"y": y.detach(), **{"d" + k: v for k, v in zip(names, grads)}})
    out = {k: torch.cat([p[k] for p in parts], 1) for k in ("y", "du", "ddt", "dz")}
    out.update({k: torch.cat([p[k] for p in parts]) for k in ("dA", "dD", "dbias")})
    out.update({k: sum(p[k] for p in parts) for k in ("dB", "dC")})
    return out
