"""Measured cases of a language model's losses over its vocabulary: the cross entropy of the logits W x, and the distillation
from a teacher's top logits, each with its gradients by x and W, without the logits being kept.

Every case is run in two forms: the plain one (elementary torch operations in 32 bits, rounded once at the end) and,
with `own` set, the library's calls.  Both see the same inputs, made on the GPU from a seed."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
MOST_FLOPS = 6 * 8192 * 65536 * 4096       # the largest listed case


# ------------------------------------------------------------------ cases
def _ce(name, op, rows, vocab, d, dtype, ignored=0.0, smoothing=0.0, z_loss=0.0, wants="xw"):
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "d": d, "dtype": dtype, "ignored": ignored, "smoothing": smoothing,
            "z_loss": z_loss, "temperature": 1.0, "wants": wants}


def _distill(name, op, rows, vocab, d, dtype, top, teacher, temperature, ignored=0.0, wants="xw"):
    return {"name": name, "op": op, "rows": rows, "vocab": vocab, "d": d, "dtype": dtype, "ignored": ignored, "top": top, "teacher": teacher,
            "temperature": temperature, "wants": wants}


def listed():
    return [
        # scores of a few held-out tokens: latency counts
        _ce("ce_few_rows", "ce", 8, 32000, 1024, "bf16"),
        # losses of a batch of 8 Ki tokens, as the reweighting of its rows reads them
        _ce("ce_batch", "ce", 8192, 65536, 4096, "bf16"),
        # a training step's gradients over the same vocabulary
        _ce("ce_batch_gradient", "ce_backward", 8192, 65536, 4096, "bf16"),
        # answers alone are trained on: six tokens of ten are left out
        _ce("ce_answers_gradient", "ce_backward", 4096, 32000, 2048, "bf16", ignored=0.6, z_loss=1e-4),
        # odd sizes in half precision, smoothed labels
        _ce("ce_odd_gradient", "ce_backward", 777, 12345, 1537, "f16", ignored=0.1, smoothing=0.1),
        # the gradients of a few tokens: bound by reading and writing the matrix
        _ce("ce_few_rows_gradient", "ce_backward", 24, 32000, 2048, "bf16"),
        # a few tokens against a teacher's 32 best
        _distill("distill_few_rows", "distill", 16, 32000, 1024, "bf16", 32, "f32", 1.0),
        # losses of a batch against a teacher's 64 best
        _distill("distill_batch", "distill", 4096, 65536, 2048, "bf16", 64, "bf16", 2.0),
        # a training step's gradients against a teacher's 128 best
        _distill("distill_batch_gradient", "distill_backward", 8192, 32000, 2048, "bf16", 128, "f32", 1.5),
        # half precision, odd sizes, the matrix is not trained
        _distill("distill_odd_gradient", "distill_backward", 1001, 5003, 515, "f16", 7, "f16", 1.0, ignored=0.2, wants="x"),
    ]


def _spread(rng, low, high):
    """A whole number spread over the logarithm of [low, high]."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def _width(rng, low, high):
    """Widths of real layers are multiples of 8, 64 or 128; one in four is odd-sized."""
    w = _spread(rng, low, high)
    step = rng.choice((1, 8, 64, 128))
    return max(step, w // step * step) if step > 1 else w


def draw(rng):
    op = rng.choice(("ce", "ce_backward", "distill", "distill_backward"))
    wants = rng.choice(("xw", "xw", "x", "w")) if op.endswith("backward") else "xw"
    while True:
        rows, vocab, d = _spread(rng, 1, 16384), _width(rng, 200, 131072), _width(rng, 64, 8192)
        if rows * vocab <= 1 << 30 and vocab * d <= 1 << 29 and _flops(op, rows, vocab, d, wants) <= MOST_FLOPS:
            break
    dtype, ignored = rng.choice(("bf16", "bf16", "f16")), rng.choice((0.0, 0.0, 0.1, 0.5, 0.9))
    if op.startswith("ce"):
        c = _ce("", op, rows, vocab, d, dtype, ignored, rng.choice((0.0, 0.0, 0.1)), rng.choice((0.0, 0.0, 1e-4)), wants)
    else:
        c = _distill("", op, rows, vocab, d, dtype, _spread(rng, 1, min(256, vocab // 2)), rng.choice(("f32", "bf16", "f16")),
                     rng.choice((1.0, 1.0, 0.7, 2.0, 4.0)), ignored, wants)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _row_blocks(rows, vocab, values):
    """Row ranges whose logits are at most `values` numbers."""
    step = max(1, values // vocab)
    return [(a, min(a + step, rows)) for a in range(0, rows, step)]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rows, vocab, d, t = case["rows"], case["vocab"], case["d"], DTYPES[case["dtype"]]

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    def uniform(*shape):
        return torch.rand(*shape, generator=g, device="cuda")

    state = dict(case, seed=seed)
    w = normal(vocab, d, scale=1.0 / math.sqrt(d)).to(t)
    x = normal(rows, d)
    keep = uniform(rows) >= case["ignored"]
    if case["op"].startswith("ce"):
        target = (vocab * uniform(rows).pow(2)).long().clamp(max=vocab - 1)      # frequent tokens have the low numbers
        x += 10.0 * uniform(rows, 1) * w[target].float()                         # some rows know their token, some do not
        state["target"] = torch.where(keep, target, -100)
    else:
        top = case["top"]
        place = torch.arange(top, device="cuda")
        step = 1 + (uniform(rows, 1) * (vocab // top - 1)).long()
        ids = ((vocab * uniform(rows, 1).pow(2)).long() + place * step) % vocab
        logits = 9.0 - 2.0 * torch.log(1.0 + place) + normal(rows, top, scale=0.5)
        for j in range(min(4, top)):
            x += (5.0 - j) * uniform(rows, 1) * w[ids[:, j]].float()
        # a tenth of the rows bring fewer entries than there is room for
        count = torch.where(uniform(rows) < 0.1, 1 + (uniform(rows) * top).long(), top)
        held = (place < count[:, None]) & keep[:, None]
        state["ids"] = torch.where(held, ids, -1).to(torch.int32)
        state["teacher"] = torch.where(held, logits, -math.inf).to(DTYPES[case["teacher"]])
    state["x"], state["w"] = x.to(t), w
    state["loss"], state["lse"] = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    if case["op"].endswith("backward"):
        state["dloss"] = 0.2 + uniform(rows) * 1.6                               # the rows' weights
        wf = w.float()
        state["lse"] = torch.cat([torch.logsumexp(state["x"][a:b].float() @ wf.t() / case["temperature"], 1) for a, b in _row_blocks(rows, vocab, 1 << 29)])
        state["lse"] = torch.where(_live(state), state["lse"], 0.0)
        state["dx"] = torch.empty_like(state["x"]) if "x" in case["wants"] else None
        state["dw"] = torch.empty_like(w) if "w" in case["wants"] else None
    return state


# ------------------------------------------------------------------ plain forms
def _live(s):
    """The rows that count: a target within the vocabulary, or an entry of the teacher's."""
    if s["op"].startswith("ce"):
        return (s["target"] >= 0) & (s["target"] < s["vocab"])
    return (_held(s)).any(1)


def _held(s):
    return (s["ids"] >= 0) & (s["ids"] < s["vocab"]) & (s["teacher"].float() > -math.inf)


def _teacher(s):
    """The teacher's distribution over its entries and its logarithm (0 where there is no entry), and the entries' places."""
    held = _held(s)
    t = torch.where(held, s["teacher"].float() / s["temperature"], -1e30)
    t = t - t.amax(1, keepdim=True)
    e = torch.where(held, torch.exp(t), 0.0)
    total = e.sum(1, keepdim=True).clamp(min=1e-30)
    return e / total, torch.where(held, t - torch.log(total), 0.0), torch.where(held, s["ids"], 0).long()


def _plain_forward(s):
    z = s["x"].float() @ s["w"].float().t() / s["temperature"]
    m = z.amax(1, keepdim=True)
    lse = (m + torch.log(torch.exp(z - m).sum(1, keepdim=True)))[:, 0]
    live = _live(s)
    if s["op"] == "ce":
        at = torch.where(live, s["target"], 0)[:, None]
        eps = s["smoothing"]
        loss = (1.0 - eps) * (lse - z.gather(1, at)[:, 0]) + eps * (lse - z.mean(1)) + s["z_loss"] * lse.square()
    else:
        p, logp, at = _teacher(s)
        loss = (p * (logp - (z.gather(1, at) - lse[:, None]))).sum(1)
    return {"loss": torch.where(live, loss, 0.0), "lse": torch.where(live, lse, 0.0)}


def _plain_backward(s):
    x, w = s["x"].float(), s["w"].float()
    live = _live(s)
    scale = torch.where(live, s["dloss"], 0.0)[:, None] / s["temperature"]
    dz = torch.exp(x @ w.t() / s["temperature"] - s["lse"][:, None])
    if s["op"] == "ce_backward":
        eps = s["smoothing"]
        dz = dz * (1.0 + 2.0 * s["z_loss"] * s["lse"])[:, None] - eps / s["vocab"]
        at, p = torch.where(live, s["target"], 0)[:, None], torch.full_like(scale, 1.0 - eps)
    else:
        p, _, at = _teacher(s)
    dz = torch.where(live[:, None], dz.scatter_add(1, at, -p) * scale, 0.0)
    out = {}
    if "x" in s["wants"]:
        out["dx"] = (dz @ w).to(s["x"].dtype)
    if "w" in s["wants"]:
        out["dw"] = (dz.t() @ x).to(s["w"].dtype)
    return out


# ------------------------------------------------------------------ one pass
def _library(s):
    """The descriptor and workspace a program keeps between its calls."""
    import paper_2207_02849_b200 as bt
    cfg = bt.VocabLoss(s["vocab"], s["d"], bt.BETTY_BF16 if s["dtype"] == "bf16" else bt.BETTY_F16, temperature=s["temperature"],
                       smoothing=s.get("smoothing", 0.0), z_loss=s.get("z_loss", 0.0))
    return bt, cfg, bt.Workspace.of_bytes(bt.betty_vocab_workspace_size(cfg, s["rows"], s.get("top", 1)))


def _own(s):
    if "library" not in s:
        s["library"] = _library(s)
    bt, cfg, ws = s["library"]
    op = s["op"]
    if op == "ce":
        bt.betty_vocab_ce(cfg, s["x"], s["w"], s["target"], s["loss"], s["lse"], ws)
    elif op == "distill":
        bt.betty_vocab_distill(cfg, s["x"], s["w"], s["ids"], s["teacher"], s["loss"], s["lse"], ws)
    elif op == "ce_backward":
        bt.betty_vocab_ce_backward(cfg, s["x"], s["w"], s["target"], s["lse"], s["dloss"], s["dx"], s["dw"], ws)
    else:
        bt.betty_vocab_distill_backward(cfg, s["x"], s["w"], s["ids"], s["teacher"], s["lse"], s["dloss"], s["dx"], s["dw"], ws)
    if not op.endswith("backward"):
        return {"loss": s["loss"], "lse": s["lse"]}
    return {"d" + k: s["d" + k] for k in s["wants"]}


def run(state):
    with torch.no_grad():
        if own:
            return _own(state)
        return _plain_backward(state) if state["op"].endswith("backward") else _plain_forward(state)


# ------------------------------------------------------------------ in 64 bits, by the definition
def exact(case, seed):
    """Row by row blocks of the logits in 64 bits; gradients by automatic differentiation of the losses."""
    s = prepare(case, seed)
    rows, vocab, backward = case["rows"], case["vocab"], case["op"].endswith("backward")
    w = s["w"].double().requires_grad_(backward)
    loss, lse = torch.zeros(rows, dtype=torch.float64, device="cuda"), torch.zeros(rows, dtype=torch.float64, device="cuda")
    dx = torch.zeros(rows, case["d"], dtype=torch.float64, device="cuda")
    for a, b in _row_blocks(rows, vocab, 1 << 28):
        with torch.enable_grad():
            x = s["x"][a:b].double().requires_grad_(backward)
            z = x @ w.t() / case["temperature"]
            some = torch.logsumexp(z, 1)
            if case["op"].startswith("ce"):
                live = s["target"][a:b] >= 0
                each = torch.nn.functional.cross_entropy(z, s["target"][a:b], ignore_index=-100, reduction="none", label_smoothing=case["smoothing"])
                each = each + case["z_loss"] * some.square() * live
            else:
                ids, there = s["ids"][a:b].long(), s["ids"][a:b] >= 0
                live = there.any(1)
                t = s["teacher"][a:b].double() / case["temperature"]
                t = torch.where(live[:, None], t, 0.0)
                logp = torch.log_softmax(t, 1)
                logq = torch.log_softmax(z, 1).gather(1, ids.clamp(min=0))
                each = torch.where(there, logp.exp() * (torch.where(there, logp, 0.0) - logq), 0.0).sum(1)
            if backward:
                each.backward(torch.where(live, s["dloss"][a:b].double(), 0.0))
                dx[a:b] = x.grad
            else:
                loss[a:b], lse[a:b] = each, torch.where(live, some, 0.0)
    if not backward:
        return {"loss": loss, "lse": lse}
    return {k: v for k, v in (("dx", dx), ("dw", w.grad)) if k[1] in case["wants"]}


# ------------------------------------------------------------------ what a pass cannot do without
def _flops(op, rows, vocab, d, wants):
    """Products of rows x vocab x d: the logits (which a backward pass has to make again), and one for each gradient."""
    return 2 * (1 + (len(wants) if op.endswith("backward") else 0)) * rows * vocab * d


def work(case):
    op, vocab, d, b = case["op"], case["vocab"], case["d"], BYTES[case["dtype"]]
    rows = max(1, round(case["rows"] * (1.0 - case["ignored"])))       # of those left out nothing has to be read but the target
    total = b * (rows * d + vocab * d) + 8 * case["rows"]
    if "top" in case:
        total += case["rows"] * case["top"] * (4 + BYTES[case["teacher"]])
    else:
        total += 8 * case["rows"]
    if op.endswith("backward"):
        total += b * d * sum({"x": case["rows"], "w": vocab}[k] for k in case["wants"])
    return {"bytes": total, "flops": _flops(op, rows, vocab, d, case["wants"])}
