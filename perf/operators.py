"""Cases of the draft head's supervised losses, measured as a training step calls them.

Three operators, each a loss with its gradient:

  xent     lmhead_cross_entropy: cross entropy of labels under logits = hidden . weight^T,
           without keeping the logits; gradients of the hidden states and of the weight.
  distill  lmhead_distill: the same LM head against a teacher's top logits,
           KL(softmax(teacher / T) || softmax(logits / T)).
  topk     topk_distill: that loss on logits in hand, with their gradient.

Every loss is the weighted mean over the counted rows: a row with an ignored
label, or with no teacher entry, is not counted (loss, log-partition and
gradient 0).  With own = False, run() computes these formulas in elementary
32-bit torch operations; with own = True it calls the library.
"""
import math

import torch

own = False

IGNORE = -100


def listed():
    """The sizes: 2*4*4 rows of 1024, 4096 rows (64*8*8) of 32000 and 4096 rows
    (32*16*8) of 128256 tokens, hidden size 4096, and odd ones around them."""
    return [
        # a debug-size step: latency of one call
        dict(name="xent small", op="xent", R=32, V=1024, H=256, ignored=0.25, weighted=False, grad=True),
        # one draft path's worth of rows against the largest vocabulary: the weight's traffic
        dict(name="xent few rows", op="xent", R=48, V=128256, H=4096, ignored=0.0, weighted=False, grad=True),
        # the draft head's training step, no row ignored
        dict(name="xent 4096x32000", op="xent", R=4096, V=32000, H=4096, ignored=0.0, weighted=True, grad=True),
        # the same over the largest vocabulary with prompt tokens ignored
        dict(name="xent 4096x128256", op="xent", R=4096, V=128256, H=4096, ignored=0.4, weighted=False, grad=True),
        # scoring held-out text: the loss alone, odd sizes
        dict(name="xent score odd", op="xent", R=1001, V=32003, H=1032, ignored=0.1, weighted=False, grad=False),
        # a debug-size distillation step
        dict(name="distill small", op="distill", R=16, V=1000, H=512, K=4, T=1.0, masked=0.0, bf16_teacher=False,
             weighted=False, grad=True),
        # a ragged batch with a warm teacher and partly filled lists
        dict(name="distill ragged", op="distill", R=777, V=32003, H=2056, K=64, T=2.0, masked=0.3, bf16_teacher=True,
             weighted=False, grad=True),
        # the draft head's distillation step, rows weighted by their depth
        dict(name="distill 4096x32000", op="distill", R=4096, V=32000, H=4096, K=10, T=1.0, masked=0.05,
             bf16_teacher=False, weighted=True, grad=True),
        # logits in hand, debug size
        dict(name="topk small", op="topk", R=32, V=1024, K=10, T=1.0, f32=True, masked=0.0, bf16_teacher=False,
             weighted=False, grad=True),
        # 16*8*6 rows of draft logits
        dict(name="topk 768x32000", op="topk", R=768, V=32000, K=32, T=1.0, f32=False, masked=0.1, bf16_teacher=True,
             weighted=True, grad=True),
        # float32 logits whose rows are not 16-byte aligned
        dict(name="topk odd f32", op="topk", R=513, V=32003, K=100, T=0.7, f32=True, masked=0.3, bf16_teacher=False,
             weighted=False, grad=True),
        # every draft row of the largest workload
        dict(name="topk 4096x128256", op="topk", R=4096, V=128256, K=10, T=1.0, f32=False, masked=0.05,
             bf16_teacher=True, weighted=True, grad=True),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(("xent", "distill", "topk"))
    while True:
        c = dict(op=op, R=_log_int(rng, 1, 6000), V=_log_int(rng, 500, 131072))
        if op == "topk":
            if c["R"] * c["V"] > 4096 * 128256:
                continue
        else:
            c["H"] = 8 * _log_int(rng, 8, 512)
            if c["R"] * c["V"] * c["H"] > 2400 * 128256 * 4096:
                continue
        break
    if op == "xent":
        c["ignored"] = rng.choice((0.0, 0.1, 0.5))
    else:
        c.update(K=_log_int(rng, 1, 128), T=rng.choice((1.0, 0.7, 2.0)), masked=rng.choice((0.0, 0.2)),
                 bf16_teacher=rng.random() < 0.5)
    if op == "topk":
        c["f32"] = rng.random() < 0.5
    c.update(weighted=rng.random() < 0.5, grad=rng.random() < 0.8)
    return c


def _teacher(case, g):
    """Top logits of a teacher, best first: a Zipf-like fall with noise; ids
    distinct in a row.  An entry that the stored list lacks has id -1 (its
    logit is whatever the buffer held, here NaN); some rows lack all of them."""
    R, V, K = case["R"], case["V"], case["K"]
    f = dict(generator=g, device="cuda")
    step = max(1, V // K)
    ids = torch.randint(0, step, (R, K), **f) + step * torch.rand(R, K, **f).argsort(1)
    t = 9.0 - 1.5 * torch.log(torch.arange(1, K + 1, device="cuda").float()) + 0.5 * torch.randn(R, K, **f)
    t = t.sort(1, descending=True).values
    if case["masked"]:
        have = torch.rand(R, 1, **f) > case["masked"] / 2
        n = torch.where(torch.rand(R, 1, **f) < case["masked"], torch.randint(1, K + 1, (R, 1), **f), K) * have
        lacks = torch.arange(K, device="cuda") >= n
        ids, t = ids.masked_fill(lacks, -1), t.masked_fill(lacks, float("nan"))
    t = t.to(torch.bfloat16) if case["bf16_teacher"] else t
    return ids.to(torch.int32), t


def _row_weights(case, g):
    """Weights by depth, 1.05^l for l = 1 .. 8, as the paths' positions have them."""
    if not case["weighted"]:
        return None
    return 1.05 ** (1.0 + torch.arange(case["R"], device="cuda") % 8).float()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    f = dict(generator=g, device="cuda")
    R, V = case["R"], case["V"]
    s = dict(case=case, row_weight=_row_weights(case, g))
    if case["op"] == "xent":
        first = labels = torch.randint(0, V, (R,), **f)
        if case["ignored"]:
            off = torch.rand(R, **f).argsort()[: int(case["ignored"] * R)]
            labels = labels.index_fill(0, off, IGNORE)
        s["labels"] = labels.to(torch.int32)
    else:
        s["ids"], s["teacher"] = _teacher(case, g)
        first = s["ids"][:, 0].long().clamp(min=0)
    if case["op"] == "topk":
        # the student: noise of its own around what it has learned of the teacher's list
        x = 2.0 * torch.randn(R, V, **f)
        x.scatter_add_(1, s["ids"].long().clamp(min=0), torch.nan_to_num(s["teacher"].float()))
        s["logits"] = x if case["f32"] else x.to(torch.bfloat16)
        return s
    H = case["H"]
    w = (0.02 * torch.randn(V, H, **f)).to(torch.bfloat16)
    # rows from untrained to confident: up to 12 on the right token's logit
    pull = 12.0 * torch.rand(R, 1, **f) / (4e-4 * H)
    s["hidden"] = (torch.randn(R, H, **f) + pull * w[first].float()).to(torch.bfloat16)
    s["weight"] = w
    return s


def _targets(s, dtype):
    """Per row the target distribution on its ids: (ids, probabilities, counted
    rows, sum p log p), in `dtype`."""
    case = s["case"]
    if case["op"] == "xent":
        lab = s["labels"].long()
        counted = lab != IGNORE
        return lab.clamp(min=0)[:, None], counted.to(dtype)[:, None], counted, torch.zeros_like(lab, dtype=dtype)
    ids = s["ids"].long()
    has = ids >= 0
    counted = has.any(1)
    t = torch.where(has, s["teacher"].to(dtype) / case["T"], float("-inf"))
    top = torch.where(counted, t.max(1).values, 0.0)[:, None]
    e = torch.exp(t - top)
    z = torch.where(counted, e.sum(1), 1.0)[:, None]
    p = e / z
    logp = torch.where(has, t - top - torch.log(z), 0.0)
    return ids.clamp(min=0), p, counted, (p * logp).sum(1)


def _plain(s):
    case, dtype = s["case"], torch.float32
    T = case.get("T", 1.0)
    ids, p, counted, plogp = _targets(s, dtype)
    if case["op"] == "topk":
        x = s["logits"].to(dtype)
    else:
        h, w = s["hidden"].to(dtype), s["weight"].to(dtype)
        x = h @ w.T
    y = x / T
    m = y.max(1).values
    logz = m + torch.log(torch.exp(y - m[:, None]).sum(1))
    rw = counted.to(dtype) if s["row_weight"] is None else s["row_weight"].to(dtype) * counted
    row_loss = torch.where(counted, plogp + logz - (p * y.gather(1, ids)).sum(1), 0.0)
    total = rw.sum()
    total = torch.where(total > 0, total, 1.0)
    out = dict(loss=((rw * row_loss).sum() / total)[None], row_loss=row_loss,
               logz=torch.where(counted, logz, 0.0))
    if case["grad"]:
        a = (rw / (total * T))[:, None]
        G = a * torch.exp(y - logz[:, None])
        G.scatter_add_(1, ids, -a * p)
        if case["op"] == "topk":
            out["grad"] = G.to(s["logits"].dtype)
        else:  # gradients have their tensors' type
            out["d_hidden"], out["d_weight"] = (G @ w).to(torch.bfloat16), (G.T @ h).to(torch.bfloat16)
    return out


def run(s):
    case = s["case"]
    if own:
        from paper_2602_05774_gb300 import vsd
        if case["op"] == "topk":
            return vsd.topk_distill(s["logits"], s["ids"], s["teacher"], T=case["T"], row_weight=s["row_weight"],
                                    grad=case["grad"])
        kw = dict(row_weight=s["row_weight"], d_hidden=case["grad"], d_weight=case["grad"])
        if case["op"] == "xent":
            return vsd.lmhead_cross_entropy(s["hidden"], s["weight"], s["labels"], ignore_index=IGNORE, **kw)
        return vsd.lmhead_distill(s["hidden"], s["weight"], s["ids"], s["teacher"], T=case["T"], **kw)
    return _plain(s)


def work(case):
    """Inputs read once, outputs written once; 2 flops a product of the counted
    rows (the logits, and with gradients the two products that carry them)."""
    R, V = case["R"], case["V"]
    small = 8 * R + (4 * R if case["weighted"] else 0)
    if case["op"] == "xent":
        rows, small = R - int(case["ignored"] * R), small + 4 * R
    else:
        rows, small = R, small + R * case["K"] * (6 if case["bf16_teacher"] else 8)
    times = 2 if case["grad"] else 1
    if case["op"] == "topk":
        return {"bytes": small + times * R * V * (4 if case["f32"] else 2), "flops": (8 if case["grad"] else 5) * R * V}
    H = case["H"]
    return {"bytes": small + times * 2 * (R * H + V * H), "flops": (6 if case["grad"] else 2) * rows * V * H}


def exact(case, seed):
    """The definition in 64 bits, row block by row block: log q_v = (x_v - x_max)
    / T - log sum exp((x - x_max) / T), L = sum_k p_k (log p_k - log q_k)."""
    s = prepare(case, seed)
    f64, T, R, V = torch.float64, case.get("T", 1.0), case["R"], case["V"]
    if case["op"] != "topk" and 6.0 * R * V * case["H"] > 1.4e13:
        return None  # the products alone take over 10 seconds in 64 bits
    if case["op"] == "xent":
        ids, t = s["labels"].long()[:, None], torch.zeros(R, 1, dtype=f64, device="cuda")
    else:
        ids, t = s["ids"].long(), s["teacher"].to(f64)
    live = ids >= 0
    wr = torch.ones(R, dtype=f64, device="cuda") if s["row_weight"] is None else s["row_weight"].to(f64)
    wr = wr * live.any(1)
    share = wr / wr.sum() if float(wr.sum()) > 0 else wr
    w = s["weight"].to(f64) if "weight" in s else None
    row_loss, logz, blocks = [], [], []
    dw = torch.zeros(V, case["H"], dtype=f64, device="cuda") if w is not None and case["grad"] else None
    for at in range(0, R, 512):
        rows = slice(at, min(R, at + 512))
        h = s["hidden"][rows].to(f64) if w is not None else None
        x = torch.matmul(h, w.t()) if w is not None else s["logits"][rows].to(f64)
        top = x.amax(1, keepdim=True)
        norm = torch.log(torch.exp((x - top) / T).sum(1, keepdim=True))
        logq = (x - top) / T - norm
        on = live[rows]
        teach = torch.where(on, t[rows] / T, torch.full_like(t[rows], -1e300))
        p = torch.softmax(teach, 1) * on
        logp = torch.where(on, torch.log_softmax(teach, 1), torch.zeros_like(teach))
        at_ids = torch.gather(logq, 1, torch.where(on, ids[rows], 0))
        row_loss.append((p * (logp - at_ids)).sum(1))
        logz.append(torch.where(on.any(1), (top / T + norm)[:, 0], torch.zeros_like(norm[:, 0])))
        if case["grad"]:
            g = torch.exp(logq)
            r, k = torch.nonzero(on, as_tuple=True)
            g.index_put_((r, ids[rows][r, k]), -p[r, k], accumulate=True)
            g *= (share[rows] / T)[:, None]
            blocks.append(g if w is None else torch.matmul(g, w))
            if dw is not None:
                dw += torch.matmul(g.t(), h)
    out = dict(loss=(share * torch.cat(row_loss)).sum()[None], row_loss=torch.cat(row_loss), logz=torch.cat(logz))
    if case["grad"]:
        out.update(dict(grad=torch.cat(blocks)) if w is None else dict(d_hidden=torch.cat(blocks), d_weight=dw))
    return out
