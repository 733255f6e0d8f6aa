"""Cases of drafting from an 8-bit head, measured as a decoding loop calls it.

Three operators that follow one another:

  quantize  quantize_fp8: a matrix in e4m3 with a power of two as scale for each
            block of 128 columns (1 row, or 128 rows, to a block).
  head      lmhead_logits_fp8: draft logits = hidden . weight^T of such matrices,
            hidden states with a scale for each row and 128 columns, the weight
            with one for each 128 x 128 block.
  sample    sample_filtered: one token a row by a given uniform number, from the
            distribution at temperature T that top-k, top-p and min-p leave; and
            filter_logits: the logits with what they leave out at -inf, as the
            verification of the drawn tokens reads them.

What is kept are the first tokens in the order of falling logits (the lower id
first among equals): the top_k first, of these as few as reach a share top_p of
their mass, and only those with at least min_p of the first one's probability.
The draw is by inverse CDF over the kept tokens in the vocabulary's order.  T = 0
keeps the first token alone.  With own = False, run() computes these formulas in
elementary torch operations (sums of probabilities, whose borders decide which
token is drawn, in 64 bits); with own = True it calls the library.
"""
import math

import torch

own = False

OFF = dict(T=1.0, top_k=0, top_p=1.0, min_p=0.0)


def listed():
    """Hidden size 4096 and vocabularies of 32000 and 128256 tokens, as in the
    benchmark's workloads, a debug size and odd ones around them."""
    return [
        # the hidden states of a training or prefill batch, every row on its own
        dict(name="quantize rows 4096x4096", op="quantize", R=4096, H=4096, block=1, f32=False),
        # a draft head's weight, once after every update of its master copy in float32
        dict(name="quantize weight 32000x4096", op="quantize", R=32000, H=4096, block=128, f32=True),
        # debug size: latency of one call
        dict(name="head small", op="head", R=32, V=1024, H=256),
        # one token each of 8 sequences against the largest vocabulary: the weight's traffic
        dict(name="head 8x128256", op="head", R=8, V=128256, H=4096),
        # a ragged batch, odd vocabulary, a last block of 16 columns
        dict(name="head ragged", op="head", R=777, V=32003, H=2064),
        # the draft logits of 64 prefixes x 8 paths x 8 positions
        dict(name="head 4096x32000", op="head", R=4096, V=32000, H=4096),
        # debug size, float32 logits, one setting for all rows
        dict(name="sample small", op="sample", R=16, V=1024, f32=True, mixed=False, T=0.8, top_k=20, top_p=0.95,
             min_p=0.05, out="token"),
        # one decoding step of 8 sequences over the largest vocabulary
        dict(name="sample 8x128256", op="sample", R=8, V=128256, f32=False, mixed=False, T=0.7, top_k=50, top_p=0.9,
             min_p=0.0, out="token"),
        # a served batch: every row has settings of its own, greedy and unfiltered ones among them
        dict(name="sample mixed 512x32000", op="sample", R=512, V=32000, f32=False, mixed=True, **OFF, out="token"),
        # the draft paths' tokens by nucleus alone, every row of the largest workload
        dict(name="sample 4096x128256", op="sample", R=4096, V=128256, f32=False, mixed=False, T=1.0, top_k=0,
             top_p=0.95, min_p=0.0, out="token"),
        # tokens and the rows they came from, float32 rows that are not 16-byte aligned
        dict(name="sample and filter odd", op="sample", R=513, V=32003, f32=True, mixed=False, T=1.0, top_k=0,
             top_p=1.0, min_p=0.05, out="both"),
        # the target's rows of a verification, filtered as the draft's were
        dict(name="filter 1024x128256", op="sample", R=1024, V=128256, f32=False, mixed=True, **OFF, out="filter"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("quantize", "head", "sample", "sample"))
    while True:
        c = dict(op=op, R=_log_int(rng, 1, 6000))
        if op == "quantize":
            c.update(R=_log_int(rng, 1, 131072), H=16 * _log_int(rng, 4, 512), block=rng.choice((1, 128)),
                     f32=rng.random() < 0.5)
            if c["R"] * c["H"] > 32000 * 4096:
                continue
        elif op == "head":
            c.update(V=_log_int(rng, 500, 131072), H=16 * _log_int(rng, 4, 512))
            if c["R"] * c["V"] * c["H"] > 4096 * 32000 * 4096:
                continue
        else:
            c.update(V=_log_int(rng, 500, 131072), f32=rng.random() < 0.5, mixed=rng.random() < 0.5, **OFF)
            if c["R"] * c["V"] > 1024 * 128256:
                continue
        break
    if op == "sample":
        if not c["mixed"]:
            c.update(T=rng.choice((0.0, 0.5, 0.7, 1.0, 1.3)), top_k=rng.choice((0, 0, 1, 10, 64, 500)),
                     top_p=rng.choice((1.0, 0.5, 0.9, 0.98)), min_p=rng.choice((0.0, 0.0, 0.03, 0.2)))
        c["out"] = rng.choice(("token", "token", "both", "filter"))
    return c


def _scale_of(amax):
    """The least power of two that takes amax / 448 to 1 at most; 1 for an empty block."""
    m, e = torch.frexp(amax / 448.0)
    s = torch.ldexp(torch.ones_like(amax), torch.where(m == 0.5, e - 1, e).clamp(-126, 127))
    return torch.where(amax > 0, s, 1.0)


def _to_blocks(x, rows):
    """[R, H] as [blocks of rows, rows, blocks of columns, 128], padded with zeros."""
    R, H = x.shape
    pad = torch.nn.functional.pad(x, (0, -H % 128, 0, -R % rows))
    return pad.reshape(pad.shape[0] // rows, rows, pad.shape[1] // 128, 128)


def _quantize(x, rows):
    """(e4m3, scales) of a matrix, one scale for each block of `rows` x 128."""
    R, H = x.shape
    b = _to_blocks(x.float(), rows)
    s = _scale_of(b.abs().amax((1, 3)))
    q = (b / s[:, None, :, None]).reshape(b.shape[0] * rows, -1)[:R, :H]
    return q.to(torch.float8_e4m3fn), s


def _spread(s, rows, R, H):
    """A scale for each element."""
    return s.repeat_interleave(rows, 0)[:R].repeat_interleave(128, 1)[:, :H]


def _logits(case, g):
    """A head of likely tokens whose logits fall with the rank's logarithm, from
    confident to open rows, over noise of all the others."""
    R, V = case["R"], case["V"]
    f = dict(generator=g, device="cuda")
    x = 1.5 * torch.randn(R, V, **f)
    n = min(V // 4, 4096)
    step = V // n
    ids = torch.randint(0, step, (R, n), **f) + step * torch.rand(R, n, **f).argsort(1)
    fall = (1.0 + 0.5 * torch.rand(R, 1, **f)) * torch.log(torch.arange(1, n + 1, device="cuda").float())
    head = 13.0 + 7.0 * torch.rand(R, 1, **f) - fall + 0.3 * torch.randn(R, n, **f)
    x.scatter_(1, ids, torch.maximum(x.gather(1, ids), head))
    return x if case["f32"] else x.to(torch.bfloat16)


def _pick(g, R, values, dtype):
    at = torch.randint(0, len(values), (R,), generator=g, device="cuda")
    return torch.tensor(values, dtype=dtype, device="cuda")[at]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    f = dict(generator=g, device="cuda")
    R = case["R"]
    if case["op"] == "quantize":
        x = torch.randn(R, case["H"], **f) * (0.02 if case["block"] > 1 else 1.0 + 3.0 * torch.rand(R, 1, **f))
        return dict(case=case, x=x if case["f32"] else x.to(torch.bfloat16))
    if case["op"] == "head":
        # rows of unlike sizes, with columns that stand out, as hidden states have them
        h = torch.randn(R, case["H"], **f) * (0.5 + torch.rand(R, 1, **f))
        h[:, :: 97] *= 8.0
        w = 0.02 * torch.randn(case["V"], case["H"], **f)
        (h8, hs), (w8, ws) = _quantize(h, 1), _quantize(w, 128)
        return dict(case=case, hidden=h8, hidden_scale=hs, weight=w8, weight_scale=ws)
    s = dict(case=case, logits=_logits(case, g), u=torch.rand(R, **f))
    if case["mixed"]:
        s.update(T=_pick(g, R, (0.0, 0.6, 0.8, 1.0, 1.0, 1.3), torch.float32),
                 top_k=_pick(g, R, (0, 0, 20, 50, 200), torch.int32),
                 top_p=_pick(g, R, (1.0, 0.8, 0.9, 0.95), torch.float32),
                 min_p=_pick(g, R, (0.0, 0.0, 0.02, 0.1), torch.float32))
    else:
        s.update({k: case[k] for k in OFF})
    return s


def _settings(s):
    """T, top_k, top_p and min_p as columns: their 32-bit values, in 64 bits."""
    dev, R = s["logits"].device, s["case"]["R"]
    cols = []
    for k in ("T", "top_k", "top_p", "min_p"):
        v = s[k]
        if not torch.is_tensor(v):
            v = torch.full((R,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device=dev)
        cols.append(v[:, None].long() if k == "top_k" else v[:, None].double())
    return cols


def _plain_sample(s):
    case, V = s["case"], s["case"]["V"]
    T, top_k, top_p, min_p = _settings(s)
    x = s["logits"].float()
    xs, order = torch.sort(x, dim=1, descending=True, stable=True)
    live = (xs > float("-inf")).sum(1, keepdim=True)
    top = xs[:, :1].double()
    Tz = torch.where(T > 0, T, 1.0)
    y = (xs.double() - top) / Tz
    e = torch.exp(y)  # falling, the first one 1
    cum = e.cumsum(1)
    k = torch.where(top_k > 0, torch.minimum(top_k, live), live)
    mass = cum.gather(1, k - 1)
    by_p = torch.where(top_p < 1, (cum < top_p * mass).sum(1, keepdim=True) + 1, V)
    by_min = torch.where(min_p > 0, (e >= min_p.clamp(max=1.0)).sum(1, keepdim=True), V)
    kept = torch.minimum(torch.minimum(k, by_p), by_min)
    kept = torch.where(T > 0, kept, 1)
    keep = torch.zeros_like(x, dtype=torch.bool).scatter_(1, order, torch.arange(V, device=x.device) < kept)
    out = dict(kept=kept[:, 0].to(torch.int32))
    if case["out"] != "token":
        out["filtered"] = torch.where(keep, s["logits"], float("-inf"))
    if case["out"] != "filter":
        y = (x.double() - top) / Tz
        c = torch.where(keep, torch.exp(y), 0.0).cumsum(1)
        z = c[:, -1:]
        tok = (c <= s["u"][:, None].double() * z).sum(1, keepdim=True)
        last = V - 1 - keep.flip(1).to(torch.int8).argmax(1, keepdim=True)
        tok = torch.minimum(tok, last)
        out["tokens"] = tok[:, 0].to(torch.int32)
        out["logq_tok"] = (y.gather(1, tok) - torch.log(z))[:, 0].float()
    return out


def run(s):
    case = s["case"]
    if own:
        from paper_2602_05774_gb300 import vsd
        if case["op"] == "quantize":
            q, scale = vsd.quantize_fp8(s["x"], block_rows=case["block"])
            return dict(q=q, scale=scale)
        if case["op"] == "head":
            return vsd.lmhead_logits_fp8(s["hidden"], s["hidden_scale"], s["weight"], s["weight_scale"])
        kw = {k: s[k] for k in OFF}
        if case["out"] == "filter":
            return vsd.filter_logits(s["logits"], **kw)
        return vsd.sample_filtered(s["logits"], s["u"], filtered=case["out"] == "both", **kw)
    if case["op"] == "quantize":
        q, scale = _quantize(s["x"], case["block"])
        return dict(q=q, scale=scale)
    if case["op"] == "head":
        R, V, H = case["R"], case["V"], case["H"]
        h = s["hidden"].float() * _spread(s["hidden_scale"], 1, R, H)
        w = s["weight"].float() * _spread(s["weight_scale"], 128, V, H)
        return (h @ w.T).to(torch.bfloat16)
    return _plain_sample(s)


def work(case):
    """Inputs read once, outputs written once; 2 flops a product, 4 a logit for
    its exponential and sums, 2 a quantized value."""
    R = case["R"]
    if case["op"] == "quantize":
        H = case["H"]
        scales = 4 * math.ceil(R / case["block"]) * math.ceil(H / 128)
        return {"bytes": R * H * ((4 if case["f32"] else 2) + 1) + scales, "flops": 2 * R * H}
    V = case["V"]
    if case["op"] == "head":
        H = case["H"]
        scales = 4 * math.ceil(H / 128) * (R + math.ceil(V / 128))
        return {"bytes": R * H + V * H + scales + 2 * R * V, "flops": 2 * R * V * H}
    size = 4 if case["f32"] else 2
    rows = R * ((16 if case["mixed"] else 0) + 4 + (12 if case["out"] != "filter" else 0))
    return {"bytes": rows + R * V * size * (1 if case["out"] == "token" else 2), "flops": 4 * R * V}


def _exact_sample(case, s):
    """Row block by row block.  The cut: the kept mass or count before each
    token, from a sort of (logit, -id)."""
    f64, V = torch.float64, case["V"]
    T, K, P, M = _settings(s)
    parts = dict(kept=[], filtered=[], tokens=[], logq_tok=[])
    for at in range(0, case["R"], 256):
        r = slice(at, min(case["R"], at + 256))
        raw = s["logits"][r]
        x = raw.to(f64)
        t, k, p, mp = T[r], K[r], P[r], M[r]
        greedy = t == 0
        best = x.amax(1, keepdim=True)
        d = x - best
        w = torch.exp(d / torch.where(greedy, torch.ones_like(t), t))
        # position of each token in the falling order
        order = torch.argsort(-x, dim=1, stable=True)
        pos = torch.empty_like(order).scatter_(1, order, torch.arange(V, device=x.device).expand_as(order))
        on = torch.isfinite(x) & ((k <= 0) | (pos < k))
        ws = torch.gather(w * on, 1, order)
        before = torch.gather(torch.cumsum(ws, 1) - ws, 1, pos)  # mass of those ahead
        total = ws.sum(1, keepdim=True)
        on &= (p >= 1) | (pos == 0) | (before < p * total)
        on &= (mp <= 0) | (w >= mp) | (d == 0)
        on &= ~greedy | (pos == 0)
        parts["kept"].append(on.sum(1).to(torch.int32))
        parts["filtered"].append(torch.where(on, x, torch.full_like(x, -math.inf)) if case["out"] != "token" else None)
        if case["out"] == "filter":
            continue
        q = w * on
        cdf = torch.cumsum(q, 1)
        z = cdf[:, -1]
        goal = s["u"][r].to(f64) * z
        tok = torch.searchsorted(cdf, goal[:, None], right=True)
        tok = torch.minimum(tok, torch.where(on, torch.arange(V, device=x.device), 0).amax(1, keepdim=True))
        parts["tokens"].append(tok[:, 0].to(torch.int32))
        parts["logq_tok"].append(torch.log(torch.gather(q, 1, tok)[:, 0] / z))
    out = dict(kept=torch.cat(parts["kept"]))
    if case["out"] != "token":
        out["filtered"] = torch.cat(parts["filtered"])
    if case["out"] != "filter":
        out.update(tokens=torch.cat(parts["tokens"]), logq_tok=torch.cat(parts["logq_tok"]))
    return out


def exact(case, seed):
    """The definitions in 64 bits."""
    s = prepare(case, seed)
    f64 = torch.float64
    if case["op"] == "sample":
        return _exact_sample(case, s)
    if case["op"] == "quantize":
        b = _to_blocks(s["x"].to(f64), case["block"])
        amax = b.abs().amax((1, 3))
        scale = torch.exp2(torch.ceil(torch.log2(amax / 448.0)))
        scale = torch.where(448.0 * scale / 2 >= amax, scale / 2, scale)  # (a logarithm a little off a whole number)
        scale = torch.where(448.0 * scale < amax, scale * 2, scale)
        scale = torch.where(amax > 0, scale, torch.ones_like(amax))
        v = (b / scale[:, None, :, None]).reshape(b.shape[0] * case["block"], -1)[: case["R"], : case["H"]]
        # e4m3: 3 bits after the leading one, the smallest exponent -6; halves to even
        step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3)
        return dict(q=torch.round(v / step) * step, scale=scale)
    R, V, H = case["R"], case["V"], case["H"]
    out = torch.zeros(R, V, dtype=f64, device="cuda")
    for k in range(0, H, 128):
        part = torch.matmul(s["hidden"][:, k : k + 128].to(f64), s["weight"][:, k : k + 128].to(f64).t())
        part *= s["hidden_scale"][:, k // 128, None].to(f64)
        part *= s["weight_scale"][:, k // 128].to(f64).repeat_interleave(128)[:V]
        out += part
    return out
