"""Measured cases of the operators of a trained residual block: its norms with gate and residual scale, the 8-bit
checkpoint of its activation, and the products of its experts, forward and backward.

Every case is run in two forms: the plain one (elementary torch operations in 32 bits, rounded once at the end) and,
with `own` set, the library's calls.  Both see the same inputs, made on the GPU from a seed."""
import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
BYTES = {"bf16": 2, "f16": 2, "f32": 4}
GROUP = 128          # values of a row that share one scale of an 8-bit checkpoint
TINY = 1e-30         # a group whose largest magnitude is below this is held as zeros


# ------------------------------------------------------------------ cases
def _norm(name, op, rows, d, x, y, norm, gate, per_gate, bias):
    return {"name": name, "op": op, "rows": rows, "d": d, "x": x, "y": y, "norm": norm, "gate": gate, "per_gate": per_gate,
            "bias": bias}


def _act(name, op, rows, cols, dtype, act, gated):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "dtype": dtype, "act": act, "gated": gated}


def _grouped(name, op, rows, spare, groups, n_in, n_out, dtype):
    return {"name": name, "op": op, "rows": rows, "spare": spare, "groups": groups, "in": n_in, "out": n_out, "dtype": dtype}


def listed():
    return [
        # one decoding step of a few sequences: latency counts
        _norm("norm_few_rows", "norm_forward", 4, 1024, "bf16", "bf16", "rms", "linear", 1, False),
        # a training batch of 16 Ki tokens, gate of every token
        _norm("norm_batch", "norm_forward", 16384, 4096, "bf16", "bf16", "rms", "sigmoid", 1, False),
        # its gradients, the gate conditioned on the sequence (one gate row per 1024 tokens)
        _norm("norm_batch_gradient", "norm_backward", 8192, 4096, "bf16", "bf16", "rms", "linear", 1024, False),
        # fp32 master activations of an odd width, layer norms with biases
        _norm("norm_odd_gradient", "norm_backward", 2731, 1537, "f32", "f32", "layer", "sigmoid", 1, True),
        # a few rows through a gated unit, checkpointed and read back
        _act("checkpoint_few_rows", "act_store", 8, 1000, "bf16", "silu", True),
        # a batch's hidden layer, checkpointed and read back
        _act("checkpoint_batch", "act_store", 16384, 4096, "bf16", "gelu", False),
        # the backward pass of a gated hidden layer from its checkpoint
        _act("checkpoint_batch_gradient", "act_backward", 8192, 8192, "f16", "silu", True),
        # fp32, odd width, last group of 5 values
        _act("checkpoint_odd_gradient", "act_backward", 777, 2053, "f32", "gelu", False),
        # two dozen tokens over eight experts: bound by reading the matrices
        _grouped("experts_few_rows", "grouped_forward", 24, 0, 8, 1024, 1024, "bf16"),
        # a training batch over eight experts
        _grouped("experts_batch", "grouped_forward", 16384, 0, 8, 4096, 4096, "bf16"),
        # gradients of the inputs: many small experts, half precision, a buffer that is not quite full
        _grouped("experts_input_gradient", "grouped_input_gradient", 5001, 119, 16, 1024, 2048, "f16"),
        # gradients of the experts' matrices
        _grouped("experts_weight_gradient", "grouped_weight_gradient", 16384, 0, 8, 2048, 4096, "bf16"),
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
    op = rng.choice(("norm_forward", "norm_backward", "act_store", "act_backward", "grouped_forward", "grouped_input_gradient",
                     "grouped_weight_gradient"))
    if op.startswith("norm"):
        d = _width(rng, 64, 8192)
        rows = _spread(rng, 1, min(16384, (1 << 25) // d))
        x, y = rng.choice((("bf16", "bf16"), ("f16", "f16"), ("f32", "f32"), ("f32", "bf16"), ("f32", "f16")))
        norm = rng.choice(("rms", "layer"))
        c = _norm("", op, rows, d, x, y, norm, rng.choice(("none", "linear", "sigmoid")), rng.choice((1, 1, 7, 128, 1000)),
                  norm == "layer" and rng.random() < 0.7)
    elif op.startswith("act"):
        cols = _width(rng, 32, 16384)
        rows = _spread(rng, 1, min(32768, (1 << 25) // cols))
        c = _act("", op, rows, cols, rng.choice(("bf16", "f16", "f32")), rng.choice(("relu", "gelu", "silu")), rng.random() < 0.5)
    else:
        n_in, n_out = _width(rng, 64, 4096), _width(rng, 64, 4096)
        rows = _spread(rng, 1, 16384)
        groups = min(_spread(rng, 1, 64), max(1, (1 << 28) // (n_in * n_out)))
        c = _grouped("", op, rows, rng.choice((0, 0, 1, 77)), groups, n_in, n_out, rng.choice(("bf16", "f16")))
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs
def _counts(rows, groups, seed):
    """Rows of each expert: uneven (weights between 1 and 3), some experts without any where rows are few."""
    r = random.Random(seed * 7919 + rows)
    if rows <= 4 * groups:
        got = [0] * groups
        for _ in range(rows):
            got[r.randrange(groups)] += 1
        return got
    w = [1.0 + 2.0 * r.random() ** 2 for _ in range(groups)]
    ends = [int(rows * sum(w[: i + 1]) / sum(w)) for i in range(groups)]
    ends[-1] = rows
    return [b - a for a, b in zip([0] + ends[:-1], ends)]


def _rows_of(state):
    """For a padded [groups, most] arrangement: the row of each place and whether it holds one, and each row's place."""
    o, most, rows = state["offsets"].long(), state["most"], state["rows"]
    at = o[:-1, None] + torch.arange(most, device="cuda")[None, :]
    held = at < o[1:, None]
    row = torch.arange(rows, device="cuda")
    group = torch.searchsorted(o, row, right=True) - 1
    used = row < o[-1]
    group = torch.where(used, group, 0)
    return at.clamp(max=rows - 1), held, group, torch.where(used, row - o[group], 0), used


def _quantise(z, cols):
    """[rows, parts * cols] in 32 bits -> whole numbers in [-127, 127] and one scale per 128 values of each part of a row."""
    rows, width = z.shape
    parts, groups = width // cols, -(-cols // GROUP)
    p = torch.nn.functional.pad(z.view(rows, parts, cols), (0, groups * GROUP - cols)).view(rows, parts * groups, GROUP)
    top = p.abs().amax(2)
    some = top >= TINY
    inv = torch.where(some, torch.reciprocal(torch.where(some, top, 1.0)) * 127.0, 0.0)
    q = torch.round(p * inv[:, :, None])
    scales = torch.where(some, top * (1.0 / 127.0), 0.0)
    return q.view(rows, parts, groups * GROUP)[:, :, :cols].reshape(rows, width), scales


def _restore(q, scales, cols):
    rows, width = q.shape
    parts, groups = width // cols, -(-cols // GROUP)
    s = scales.view(rows, parts, groups).repeat_interleave(GROUP, 2)[:, :, :cols].reshape(rows, width)
    return q.float() * s


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    op = case["op"]

    def normal(*shape, dtype=torch.float32, scale=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * scale).to(dtype)

    state = dict(case, seed=seed, gate_kind=case.get("gate"))
    if op.startswith("norm"):
        rows, d, tx, ty = case["rows"], case["d"], DTYPES[case["x"]], DTYPES[case["y"]]
        gates = -(-rows // case["per_gate"])
        n = 5 if case["bias"] else 3
        params = normal(n, d, scale=0.1)      # [w_pre, w_post, residual scale (, b_pre, b_post)]
        params[:2] += 1.0
        params[2] += 0.5
        state["params"] = params
        state["y"] = normal(rows, d, dtype=ty, scale=0.7) + 0.1
        state["gate"] = normal(gates, d, dtype=ty) if case["gate"] != "none" else None
        if op == "norm_forward":
            state["x_in"] = normal(rows, d, dtype=tx, scale=2.0)
            state["x_out"], state["u"] = torch.empty_like(state["x_in"]), torch.empty_like(state["y"])
        else:
            state["x_out"] = normal(rows, d, dtype=tx, scale=2.0)
            state["du"], state["dx_out"] = normal(rows, d, dtype=ty), normal(rows, d, dtype=tx)
            state["dx"], state["dy"] = torch.empty_like(state["x_out"]), torch.empty_like(state["y"])
            state["dgate"] = torch.empty_like(state["gate"]) if state["gate"] is not None else None
            state["dparams"] = torch.empty_like(params)
    elif op.startswith("act"):
        rows, cols, t = case["rows"], case["cols"], DTYPES[case["dtype"]]
        width = cols * (2 if case["gated"] else 1)
        z = normal(rows, width, scale=1.2)
        z[:, :: 61] *= 4.0                    # a few wide channels, as hidden layers have
        z = z.to(t)
        groups = width // cols * -(-cols // GROUP)
        if op == "act_store":
            state["z"], state["a"], state["back"] = z, torch.empty(rows, cols, dtype=t, device="cuda"), torch.empty_like(z)
            state["q"] = torch.empty(rows, width, dtype=torch.int8, device="cuda")
            state["scales"] = torch.empty(rows, groups, device="cuda")
        else:
            q, state["scales"] = _quantise(z.float(), cols)
            state["q"] = q.to(torch.int8)
            state["da"] = normal(rows, cols, dtype=t)
            state["dz"], state["a"] = torch.empty_like(z), torch.empty(rows, cols, dtype=t, device="cuda")
    else:
        rows, t, e, n_in, n_out = case["rows"] + case["spare"], DTYPES[case["dtype"]], case["groups"], case["in"], case["out"]
        counts = _counts(case["rows"], e, seed)
        offsets = [0]
        for c in counts:
            offsets.append(offsets[-1] + c)
        state["rows"], state["most"] = rows, max(counts)
        state["offsets"] = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        if op != "grouped_weight_gradient":
            state["w"] = normal(e, n_out, n_in, dtype=t, scale=1.0 / math.sqrt(n_in))
        if op != "grouped_input_gradient":
            state["x"] = normal(rows, n_in, dtype=t)
        if op != "grouped_forward":
            state["dy"] = normal(rows, n_out, dtype=t, scale=0.1)
        state["result"] = torch.empty({"grouped_forward": (rows, n_out), "grouped_input_gradient": (rows, n_in),
                                       "grouped_weight_gradient": (e, n_out, n_in)}[op], dtype=t, device="cuda")
    return state


# ------------------------------------------------------------------ plain forms
def _normed(v, kind, eps):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    r = torch.rsqrt(v.square().mean(1, keepdim=True) + eps)
    return v * r, r


def _norm_back(dn, n, r, kind):
    dv = dn - n * (dn * n).mean(1, keepdim=True)
    if kind == "layer":
        dv = dv - dn.mean(1, keepdim=True)
    return dv * r


EPS = 1e-6


def _gate_rows(state):
    """The gate of each row as it multiplies, and its derivative by the gate's own value."""
    rows, per = state["rows"], state["per_gate"]
    if state["gate_kind"] == "none":
        return 1.0, None
    v = state["gate"].float()
    if per > 1:
        v = v.repeat_interleave(per, 0)[:rows]
    if state["gate_kind"] == "linear":
        return v, 1.0
    s = torch.sigmoid(v)
    return s, s * (1.0 - s)


def _plain_norm_forward(s):
    p = s["params"]
    a, _ = _gate_rows(s)
    z = _normed(s["y"].float(), s["norm"], EPS)[0] * p[1]
    if s["bias"]:
        z = z + p[4]
    x_out = s["x_in"].float() + p[2] * a * z
    u = _normed(x_out, s["norm"], EPS)[0] * p[0]
    if s["bias"]:
        u = u + p[3]
    return {"x_out": x_out.to(s["x_in"].dtype), "u": u.to(s["y"].dtype)}


def _plain_norm_backward(s):
    p, rows, per = s["params"], s["rows"], s["per_gate"]
    du = s["du"].float()
    n, r = _normed(s["x_out"].float(), s["norm"], EPS)
    dx = s["dx_out"].float() + _norm_back(du * p[0], n, r, s["norm"])
    a, da = _gate_rows(s)
    m, q = _normed(s["y"].float(), s["norm"], EPS)
    dy = _norm_back(dx * p[2] * a * p[1], m, q, s["norm"])
    d_post = (dx * a * m).sum(0)
    grads = [(du * n).sum(0), p[2] * d_post, p[1] * d_post]
    if s["bias"]:
        d_bias = (dx * a).sum(0)
        grads[2] = grads[2] + p[4] * d_bias
        grads += [du.sum(0), p[2] * d_bias]
    out = {"dx": dx.to(s["x_out"].dtype), "dy": dy.to(s["y"].dtype), "dparams": torch.stack(grads)}
    if s["gate_kind"] != "none":
        z = m * p[1] + p[4] if s["bias"] else m * p[1]
        dg = dx * p[2] * z * da
        if per > 1:
            dg = torch.nn.functional.pad(dg, (0, 0, 0, -rows % per)).view(-1, per, s["d"]).sum(1)
        out["dgate"] = dg.to(s["y"].dtype)
    return out


def _act_and_slope(v, kind):
    if kind == "relu":
        on = (v > 0).float()
        return v * on, on
    if kind == "silu":
        s = torch.sigmoid(v)
        return v * s, s * (1.0 + v * (1.0 - s))
    cdf = 0.5 * (1.0 + torch.erf(v * math.sqrt(0.5)))
    return v * cdf, cdf + v * torch.exp(-0.5 * v * v) * (1.0 / math.sqrt(2.0 * math.pi))


def _plain_act_store(s):
    z, cols = s["z"].float(), s["cols"]
    a = _act_and_slope(z[:, :cols], s["act"])[0]
    if s["gated"]:
        a = a * z[:, cols:]
    q, scales = _quantise(z, cols)
    return {"a": a.to(s["z"].dtype), "back": _restore(q, scales, cols).to(s["z"].dtype)}


def _plain_act_backward(s):
    cols, t = s["cols"], s["da"].dtype
    z, da = _restore(s["q"], s["scales"], cols), s["da"].float()
    a, slope = _act_and_slope(z[:, :cols], s["act"])
    if not s["gated"]:
        return {"dz": (da * slope).to(t), "a": a.to(t)}
    v = z[:, cols:]
    return {"dz": torch.cat((da * v * slope, da * a), 1).to(t), "a": (a * v).to(t)}


def _plain_grouped(s):
    at, held, group, place, used = _rows_of(s)
    op, t = s["op"], DTYPES[s["dtype"]]
    if op == "grouped_weight_gradient":
        keep = held[:, :, None].float()
        return {"dw": torch.bmm((s["dy"].float()[at] * keep).transpose(1, 2), s["x"].float()[at] * keep).to(t)}
    if op == "grouped_forward":
        p = torch.bmm(s["x"].float()[at], s["w"].float().transpose(1, 2))
    else:
        p = torch.bmm(s["dy"].float()[at], s["w"].float())
    p = torch.where(used[:, None], p[group, place], 0.0).to(t)
    return {"y" if op == "grouped_forward" else "dx": p}


# ------------------------------------------------------------------ one pass
def _library(s):
    """The descriptor and workspace a program keeps between its calls."""
    import paper_2207_02849_b200 as bt
    op = s["op"]
    if op.startswith("norm"):
        kind = {"rms": bt.NORM_RMS, "layer": bt.NORM_LAYER}[s["norm"]]
        cfg = bt.BlockNorm(s["d"], pre=kind, post=kind, gate={"none": bt.GATE_NONE, "linear": bt.GATE_LINEAR, "sigmoid": bt.GATE_SIGMOID}[s["gate_kind"]],
                           rows_per_gate=s["per_gate"], eps=EPS, bias=s["bias"])
        ws = bt.Workspace.of_bytes(bt.betty_block_norm_workspace_size(cfg, s["rows"])) if op == "norm_backward" else None
    elif op.startswith("act"):
        cfg = bt.Act8(s["cols"], act={"relu": bt.ACT_RELU, "gelu": bt.ACT_GELU, "silu": bt.ACT_SILU}[s["act"]], gated=s["gated"])
        ws = None
    else:
        cfg = bt.Grouped(s["groups"], s["in"], s["out"], bt.BETTY_BF16 if s["dtype"] == "bf16" else bt.BETTY_F16)
        ws = bt.Workspace.of_bytes(bt.betty_grouped_workspace_size(cfg, s["rows"]))
    return bt, cfg, ws


def _own(s):
    if "library" not in s:
        s["library"] = _library(s)
    bt, cfg, ws = s["library"]
    op = s["op"]
    if op == "norm_forward":
        bt.betty_block_norm(cfg, s["params"], s["x_in"], s["y"], s["gate"], s["x_out"], s["u"])
        return {"x_out": s["x_out"], "u": s["u"]}
    if op == "norm_backward":
        bt.betty_block_norm_backward(cfg, s["params"], s["x_out"], s["y"], s["gate"], s["du"], s["dx_out"], s["dx"], s["dy"], s["dgate"],
                                     s["dparams"], ws)
        out = {"dx": s["dx"], "dy": s["dy"], "dparams": s["dparams"]}
        if s["dgate"] is not None:
            out["dgate"] = s["dgate"]
        return out
    if op == "act_store":
        bt.betty_act8_store(cfg, s["z"], s["a"], s["q"], s["scales"])
        bt.betty_act8_restore(cfg, s["q"], s["scales"], s["back"])
        return {"a": s["a"], "back": s["back"]}
    if op == "act_backward":
        bt.betty_act8_backward(cfg, s["q"], s["scales"], s["da"], s["dz"], s["a"])
        return {"dz": s["dz"], "a": s["a"]}
    if op == "grouped_forward":
        bt.betty_grouped_forward(cfg, s["offsets"], s["x"], s["w"], s["result"], ws)
        return {"y": s["result"]}
    if op == "grouped_input_gradient":
        bt.betty_grouped_backward_data(cfg, s["offsets"], s["dy"], s["w"], s["result"], ws)
        return {"dx": s["result"]}
    bt.betty_grouped_backward_weight(cfg, s["offsets"], s["dy"], s["x"], s["result"], ws)
    return {"dw": s["result"]}


PLAIN = {"norm_forward": _plain_norm_forward, "norm_backward": _plain_norm_backward, "act_store": _plain_act_store,
         "act_backward": _plain_act_backward, "grouped_forward": _plain_grouped, "grouped_input_gradient": _plain_grouped,
         "grouped_weight_gradient": _plain_grouped}


def run(state):
    with torch.no_grad():
        return _own(state) if own else PLAIN[state["op"]](state)


# ------------------------------------------------------------------ what a pass cannot do without
def work(case):
    op = case["op"]
    if op.startswith("norm"):
        n, x, y = case["rows"] * case["d"], BYTES[case["x"]], BYTES[case["y"]]
        gates = -(-case["rows"] // case["per_gate"]) * case["d"] * y if case["gate"] != "none" else 0
        params = (5 if case["bias"] else 3) * case["d"] * 4
        if op == "norm_forward":
            return {"bytes": n * (2 * x + 2 * y) + gates + params, "flops": 20 * n}
        return {"bytes": n * (3 * x + 3 * y) + 2 * gates + 2 * params, "flops": 40 * n}
    if op.startswith("act"):
        n, b, parts = case["rows"] * case["cols"], BYTES[case["dtype"]], 2 if case["gated"] else 1
        scales = case["rows"] * parts * -(-case["cols"] // GROUP) * 4
        # store and read back: z in, a out, the checkpoint out and in, its values out; backward: the checkpoint and da in, dz and a out
        total = n * (parts * (2 * b + 2) + b) + 2 * scales if op == "act_store" else n * (parts * (1 + b) + 2 * b) + scales
        return {"bytes": total, "flops": 20 * n * parts}
    rows, e, n_in, n_out = case["rows"], case["groups"], case["in"], case["out"]
    used = min(e, rows)
    return {"bytes": 2 * ((rows + case["spare"]) * (n_in + n_out) + (e if op == "grouped_weight_gradient" else used) * n_in * n_out),
            "flops": 2 * rows * n_in * n_out}


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    host = lambda v: {k: x.cpu() for k, x in v.items()}  # noqa: E731
    if op.startswith("norm"):
        return host(_exact_norm(s))
    if op.startswith("act"):
        return host(_exact_act(s))
    o, result = s["offsets"].tolist(), []
    for e in range(s["groups"]):
        a, b = o[e], o[e + 1]
        if op == "grouped_forward":
            result.append(s["x"][a:b].double() @ s["w"][e].double().t())
        elif op == "grouped_input_gradient":
            result.append(s["dy"][a:b].double() @ s["w"][e].double())
        else:
            result.append(s["dy"][a:b].double().t() @ s["x"][a:b].double())
    if op == "grouped_weight_gradient":
        return host({"dw": torch.stack(result)})
    got = torch.cat(result)
    rest = torch.zeros(s["rows"] - o[-1], got.shape[1], dtype=torch.float64, device="cuda")
    return host({"y" if op == "grouped_forward" else "dx": torch.cat((got, rest))})


def _exact_norm(s):
    d, kind, bias = s["d"], s["norm"], s["bias"]
    leaf = lambda t: t.double().detach().requires_grad_(True)  # noqa: E731
    par = [leaf(row) for row in s["params"]]
    y = leaf(s["y"])
    gate = leaf(s["gate"]) if s["gate"] is not None else None

    def unit(v):
        if kind == "layer":
            return torch.nn.functional.layer_norm(v, (d,), eps=EPS)
        return v / (v.pow(2).sum(1, keepdim=True) / d + EPS).sqrt()

    def entry(x):
        return unit(x) * par[0] + (par[3] if bias else 0.0)

    def change():
        z = unit(y) * par[1] + (par[4] if bias else 0.0)
        if gate is not None:
            rows = gate[torch.arange(s["rows"], device="cuda") // s["per_gate"]]
            z = z * (rows if s["gate_kind"] == "linear" else 1.0 / (1.0 + torch.exp(-rows)))
        return par[2] * z

    if s["op"] == "norm_forward":
        with torch.no_grad():
            x = s["x_in"].double() + change()
            return {"x_out": x, "u": entry(x)}
    with torch.enable_grad():
        x = leaf(s["x_out"])
        first = [x, par[0]] + ([par[3]] if bias else [])
        got = torch.autograd.grad(entry(x), first, s["du"].double())
        dx = got[0] + s["dx_out"].double()
        second = [y, par[1], par[2]] + ([gate] if gate is not None else []) + ([par[4]] if bias else [])
        more = torch.autograd.grad(change(), second, dx)
    out = {"dx": dx, "dy": more[0], "dparams": torch.stack([got[1], more[1], more[2]] + ([got[2], more[-1]] if bias else []))}
    if gate is not None:
        out["dgate"] = more[3]
    return out


def _exact_act(s):
    cols, kind = s["cols"], s["act"]

    def act(v):
        if kind == "relu":
            return v.clamp(min=0.0)
        if kind == "silu":
            return v / (1.0 + torch.exp(-v))
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2.0))

    def unit(z):
        return act(z[:, :cols]) * z[:, cols:] if s["gated"] else act(z)

    def blocks(v):
        return [(p + k, min(p + k + GROUP, p + cols)) for p in range(0, v.shape[1], cols) for k in range(0, cols, GROUP)]

    if s["op"] == "act_store":
        z = s["z"].double()
        back = torch.empty_like(z)
        for a, b in blocks(z):
            top = z[:, a:b].abs().max(1, keepdim=True)[0]
            step = top / 127.0
            back[:, a:b] = torch.where(top >= TINY, torch.round(z[:, a:b] / step.clamp(min=1e-300)) * step, 0.0)
        return {"a": unit(z), "back": back}
    z = s["q"].double()
    for i, (a, b) in enumerate(blocks(z)):
        z[:, a:b] *= s["scales"][:, i : i + 1].double()
    with torch.enable_grad():
        z = z.requires_grad_(True)
        a = unit(z)
        (dz,) = torch.autograd.grad(a, z, s["da"].double())
    return {"dz": dz, "a": a.detach()}
