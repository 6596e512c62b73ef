"""Operators next to the MoE block, timed one pass at a time: products in 8-bit floating point with a scale for each
block of 128, over one matrix, over the experts of a grouping and inside the block; the balance loss of the gate and its
backward pass.  ``own`` False: plain torch operations in 32 bits.  ``own`` True: the calls of the framework.
"""
import math

import torch

own = False

GROUP = 128                        # columns (and rows, for weights) that share a scale
TOP = 448.0                        # largest e4m3 value
SIGMA_W = 0.02                     # the weights of this repository's workloads
F8 = torch.float8_e4m3fn


# ---------------------------------------------------------------- cases

def _product(name, n, inn, out, y):
    return dict(name=name, op="product", n=n, inn=inn, out=out, y=y)


def _grouped(name, T, E, k, inn, out, y, spread):
    return dict(name=name, op="grouped", T=T, E=E, k=k, inn=inn, out=out, y=y, spread=spread)


def _block(name, T, d, f, E, k):
    return dict(name=name, op="block", T=T, d=d, f=f, E=E, k=k)


def _loss(name, T, E, k, padded):
    return dict(name=name, op="loss", T=T, E=E, k=k, padded=padded)


def _backward(name, T, d, E, k, padded, dx):
    return dict(name=name, op="backward", T=T, d=d, E=E, k=k, padded=padded, dx=dx)


def listed():
    return [
        # one token through one projection of the Mixtral shape: a read of the weights
        _product("product_one_row", 1, 4096, 14336, "f16"),
        # a handful of rows, a width that ends inside a block and an odd number of outputs
        _product("product_few_ragged", 37, 1488, 1001, "f32"),
        # a long prompt through the same projection: bound by the matrix cores
        _product("product_prompt", 4096, 4096, 14336, "f16"),
        # the gradient with respect to the rows: g times the matrix, through its transposed codes
        _product("gradient_rows", 1000, 14336, 4096, "f32"),
        # the up-projection of a prompt's pairs over 8 experts, rows gathered from the tokens
        _grouped("experts_prompt", 2048, 8, 2, 4096, 14336, "f16", 0.0),
        # many small experts, a skewed load, some of them without a row
        _grouped("experts_skewed", 300, 32, 4, 2048, 1408, "f32", 1.2),
        # the whole block with experts of this form: decode and a prompt
        _block("block_one_token", 1, 4096, 14336, 8, 2),
        _block("block_prompt", 512, 4096, 14336, 8, 2),
        # the balance loss of a serving batch that is watched, and of a training batch with padding
        _loss("loss_small", 16, 8, 2, 0.0),
        _loss("loss_training", 65536, 32, 4, 0.2),
        # the backward pass of the gate for a small batch and for a training batch with padding
        _backward("backward_small", 333, 1024, 8, 2, 0.1, "f32"),
        _backward("backward_training", 16384, 4096, 32, 4, 0.1, "f16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["product", "product", "grouped", "block", "loss", "backward"])
    y = rng.choice(["f16", "f32"])
    if op == "product":
        while True:
            n, inn, out = _log(rng, 1, 4096), 16 * _log(rng, 4, 1024), _log(rng, 17, 16384)
            if n * inn * out <= 4096 * 4096 * 14336 / 2:
                return dict(op=op, n=n, inn=inn, out=out, y=y)
    if op == "grouped":
        E = rng.randint(2, 32)
        k = rng.randint(1, min(E, 8))
        while True:
            T, inn, out = _log(rng, 1, 2048), 16 * _log(rng, 8, 512), _log(rng, 100, 8192)
            if E * inn * out <= 8 * 4096 * 14336 and T * k * inn * out <= 4096 * 4096 * 14336 / 2:
                return dict(op=op, T=T, E=E, k=k, inn=inn, out=out, y=y, spread=rng.choice([0.0, 1.2]))
    if op == "block":
        E = rng.randint(2, 16)
        while True:
            T, d, f = _log(rng, 1, 512), 64 * _log(rng, 8, 64), 64 * _log(rng, 16, 224)
            if E * d * f <= 8 * 4096 * 14336:
                return dict(op=op, T=T, d=d, f=f, E=E, k=rng.randint(1, min(E, 4)))
    E = rng.randint(2, 32)
    k, padded = rng.randint(1, min(E, 8)), rng.choice([0.0, 0.1, 0.3])
    if op == "loss":
        return dict(op=op, T=_log(rng, 2, 65536), E=E, k=k, padded=padded)
    return dict(op=op, T=_log(rng, 2, 16384), d=64 * _log(rng, 4, 64), E=E, k=k, padded=padded, dx=y)


# ---------------------------------------------------------------- inputs

def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _normal(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).half()


def _blocks(w):
    """[..., out, in] padded with zeros to whole blocks, as [..., out/128, 128, in/128, 128]."""
    out, inn = w.shape[-2:]
    w = torch.nn.functional.pad(w, (0, -inn % GROUP, 0, -out % GROUP))
    return w.reshape(*w.shape[:-2], w.shape[-2] // GROUP, GROUP, w.shape[-1] // GROUP, GROUP)


def _matrix(g, out, inn):
    """Codes and scales of a weight matrix, quantized once and kept."""
    b = _blocks(_normal(g, out, inn, scale=SIGMA_W).float())
    most = b.abs().amax((1, 3), keepdim=True)
    codes = (b * (torch.full_like(most, TOP) / most)).to(F8).reshape(b.shape[0] * GROUP, b.shape[2] * GROUP)
    scale = (most / torch.full_like(most, TOP)).reshape(b.shape[0], b.shape[2])
    return codes[:out, :inn].contiguous(), scale.contiguous()


def _outputs(n, inn, rows, out, y):
    """Where the calls put quantized rows and the product."""
    return dict(codes=torch.empty(n, inn, dtype=F8, device="cuda"),
                scale=torch.empty(-(-inn // GROUP), n, device="cuda"),
                y=torch.empty(rows, out, dtype=torch.float16 if y == "f16" else torch.float32, device="cuda"))


def _choices(g, T, E, k, spread):
    """k different experts per token, the first ones in demand if spread > 0, and the grouping of the pairs by expert."""
    taste = torch.randn(T, E, generator=g, device="cuda") - 2 * spread * torch.log(torch.arange(1, E + 1, device="cuda"))
    idx = taste.topk(k, 1).indices.int()
    perm = torch.sort(idx.reshape(-1), stable=True).indices.int()
    counts = torch.bincount(idx.reshape(-1), minlength=E)
    offsets = torch.cat([torch.zeros(1, dtype=torch.int64, device="cuda"), counts.cumsum(0)]).int()
    return idx, perm, offsets, counts.tolist()


def _clear_tokens(g, w_gate, T, d, k):
    """Tokens whose choice of k experts does not hang on the last bits of a logit."""
    x = _normal(g, 2 * T + 64, d)
    logits = (x.double() @ w_gate.double().t()).sort(1, descending=True).values
    gap = (logits[:, : k] - logits[:, 1: k + 1]).amin(1) if w_gate.shape[0] > k else logits[:, 0] * 0 + 1
    return x[(gap < 1e-4).int().sort(stable=True).indices[:T]].contiguous()


def prepare(case, seed):
    g, op = _generator(seed), case["op"]
    s = dict(case)
    if op in ("product", "grouped"):
        n = case["n"] if op == "product" else case["T"]
        s["x"] = _normal(g, n, case["inn"])
        s["w"] = [_matrix(g, case["out"], case["inn"]) for _ in range(case.get("E", 1))]
        rows = n
        if op == "grouped":
            _, s["perm"], s["offsets"], s["counts"] = _choices(g, n, case["E"], case["k"], case["spread"])
            rows = n * case["k"]
        s |= _outputs(n, case["inn"], rows, case["out"], case["y"])
    elif op == "block":
        T, d, f, E = case["T"], case["d"], case["f"], case["E"]
        s["w_gate"] = _normal(g, E, d, scale=SIGMA_W)
        s["x"] = _clear_tokens(g, s["w_gate"], T, d, case["k"])
        s["experts"] = [[_matrix(g, f, d), _matrix(g, f, d), _matrix(g, d, f)] for _ in range(E)]
        s["out"] = torch.empty(T, d, dtype=torch.float16, device="cuda")
    else:
        T, E, k = case["T"], case["E"], case["k"]
        s["logits"] = torch.randn(T, E, generator=g, device="cuda") * 1.3
        s["idx"] = s["logits"].topk(k, 1).indices.int()
        s["valid"] = None
        if case["padded"]:
            s["valid"] = (torch.rand(T, generator=g, device="cuda") >= case["padded"]).to(torch.uint8)
            s["valid"][0] = 1
        new = lambda *shape, t=torch.float32: torch.empty(*shape, dtype=t, device="cuda")  # noqa: E731
        if op == "loss":
            s |= dict(counts=new(E + 1, t=torch.int32), mean_prob=new(E), loss=new(1))
        else:
            d = case["d"]
            s["x"], s["w_gate"] = _normal(g, T, d), _normal(g, E, d, scale=SIGMA_W)
            valid = torch.ones(T, dtype=torch.uint8, device="cuda") if s["valid"] is None else s["valid"]
            pairs = torch.where(valid[:, None] > 0, s["idx"], E).reshape(-1)
            s["counts"] = torch.bincount(pairs, minlength=E + 1).int()
            s["counts"][E] = valid.int().sum()
            s["d_gate"] = torch.randn(T, k, generator=g, device="cuda")
            s["d_loss"] = torch.full((1,), 0.01 * T, device="cuda")   # a loss over tokens, scaled against underflow
            s |= dict(d_logits=new(T, E), d_w_gate=new(E, d), d_bias=new(E),
                      d_x=new(T, d, t=torch.float16 if case["dx"] == "f16" else torch.float32))
    if own:
        _keep(s)
    return s


# ---------------------------------------------------------------- the framework's calls

def _keep(s):
    """The descriptors and workspaces that a program builds once."""
    from paper_2407_14417_amd import binding as mm
    s["mm"] = mm
    if s["op"] in ("product", "grouped"):
        s["mats"] = [mm.Mat(c, z) for c, z in s["w"]]
        if s["op"] == "grouped":
            s["mats"] = mm.MatGroup(s["mats"])
        return
    if s["op"] == "block":
        experts = [mm.Expert(mm.PREC_FP8B128, *[mm.Mat(c, z) for c, z in e]) for e in s["experts"]]
        s["layer"] = mm.Layer(s["d"], s["f"], s["k"], s["w_gate"], experts)
        s["ws"] = mm.alloc_workspace(s["layer"], s["T"])
        return
    d = s.get("d", 64)
    gate = s["w_gate"] if "w_gate" in s else torch.zeros(s["E"], d, dtype=torch.float16, device="cuda")
    experts = [mm.Expert(mm.PREC_FP16, None, None, None, resident=False) for _ in range(s["E"])]
    s["layer"] = mm.Layer(d, 64, s["k"], gate, experts)
    s["ws"] = mm.alloc_gate_workspace(s["layer"], s["T"])


def _run_own(s):
    mm, op = s["mm"], s["op"]
    if op == "block":
        mm.moe_layer_forward(s["layer"], s["x"], s["out"], s["ws"])
        return dict(out=s["out"])
    if op == "loss":
        mm.moe_balance_loss(s["layer"], s["logits"], s["idx"], s["counts"], s["mean_prob"], s["loss"], s["ws"], valid=s["valid"])
        return dict(counts=s["counts"], mean_prob=s["mean_prob"], loss=s["loss"])
    if op == "backward":
        mm.moe_route_backward(s["layer"], s["x"], s["logits"], s["idx"], s["ws"], valid=s["valid"], counts=s["counts"],
                              d_gate=s["d_gate"], d_loss=s["d_loss"], d_logits=s["d_logits"], d_x=s["d_x"],
                              d_w_gate=s["d_w_gate"], d_bias=s["d_bias"])
        return dict(d_logits=s["d_logits"], d_x=s["d_x"], d_w_gate=s["d_w_gate"], d_bias=s["d_bias"])
    mm.moe_quantize_fp8_rows(s["x"], s["codes"], s["scale"])
    if op == "product":
        mm.moe_matmul_fp8(s["mats"][0], s["codes"], s["scale"], s["y"])
    else:
        mm.moe_matmul_fp8_grouped(s["mats"], s["codes"], s["scale"], s["offsets"], s["perm"], s["k"], s["y"])
    return dict(codes=s["codes"], scale=s["scale"], y=s["y"])


# ---------------------------------------------------------------- plain forms, 32 bits

def _quantize_rows(x):
    n, inn = x.shape
    b = torch.nn.functional.pad(x.float(), (0, -inn % GROUP)).reshape(n, -1, GROUP)
    most = b.abs().amax(2, keepdim=True)
    top = torch.full_like(most, TOP)
    codes = (b * torch.where(most > 0, top / most, 0)).to(F8).reshape(n, -1)[:, :inn]
    return codes.contiguous(), (most / top)[:, :, 0].t().contiguous()


def _rows_of(codes, scale):
    """Quantized rows as the fp32 values they stand for."""
    return codes.float() * scale.t().repeat_interleave(GROUP, 1)[:, : codes.shape[1]]


def _weights_of(w):
    codes, scale = w
    b = _blocks(codes.float()) * scale[:, None, :, None]
    return b.reshape(b.shape[0] * GROUP, -1)[: codes.shape[0], : codes.shape[1]]


def _each_expert(rows, weights, counts):
    """The products of an expert's rows with its matrix, experts one after the other, those with rows alone."""
    parts = rows.split(counts)
    return torch.cat([p @ _weights_of(w).t() for p, w in zip(parts, weights) if p.shape[0]])


def _run_block(s):
    x, k = s["x"].float(), s["k"]
    logits, idx = (x @ s["w_gate"].float().t()).topk(k, 1)
    gates = torch.softmax(logits, 1)
    perm = torch.sort(idx.reshape(-1), stable=True).indices
    counts = torch.bincount(idx.reshape(-1), minlength=s["E"]).tolist()
    rows = _rows_of(*_quantize_rows(s["x"]))[perm // k]
    up, gate = (_each_expert(rows, [e[i] for e in s["experts"]], counts) for i in (1, 0))
    h = (gate / (1 + torch.exp(-gate)) * up).half()
    y = _each_expert(_rows_of(*_quantize_rows(h)), [e[2] for e in s["experts"]], counts)
    pairs = torch.empty_like(y)
    pairs[perm] = y
    return dict(out=(pairs.reshape(-1, k, y.shape[1]) * gates[:, :, None]).sum(1).half())


def _run_loss(s):
    E, k = s["E"], s["k"]
    p = torch.softmax(s["logits"], 1)
    one = torch.zeros_like(p).scatter_(1, s["idx"].long(), 1.0)
    n = torch.tensor(float(s["T"]), device="cuda")
    if s["valid"] is not None:
        p, one, n = p * s["valid"][:, None], one * s["valid"][:, None], s["valid"].sum().float()
    counts, mean = one.sum(0), p.sum(0) / n
    loss = (counts * mean).sum() * E / (n * k)
    return dict(counts=torch.cat([counts, n[None]]).int(), mean_prob=mean, loss=loss[None])


def _run_backward(s):
    E, k, idx = s["E"], s["k"], s["idx"].long()
    c, n = s["counts"][:E].float(), s["counts"][E].float()
    p = torch.softmax(s["logits"], 1)
    dl = p * (c - (p * c).sum(1, keepdim=True)) * (s["d_loss"] * E / (n * n * k))
    gates = torch.softmax(s["logits"].gather(1, idx), 1)
    dl = dl.scatter_add(1, idx, gates * (s["d_gate"] - (gates * s["d_gate"]).sum(1, keepdim=True)))
    if s["valid"] is not None:
        dl = dl * s["valid"][:, None]
    x, w = s["x"].float(), s["w_gate"].float()
    return dict(d_logits=dl, d_x=(dl @ w).to(s["d_x"].dtype), d_w_gate=dl.t() @ x, d_bias=dl.sum(0))


def run(state):
    if own:
        return _run_own(state)
    op = state["op"]
    if op in ("block", "loss", "backward"):
        return {"block": _run_block, "loss": _run_loss, "backward": _run_backward}[op](state)
    codes, scale = _quantize_rows(state["x"])
    rows = _rows_of(codes, scale)
    if op == "product":
        y = rows @ _weights_of(state["w"][0]).t()
    else:
        y = _each_expert(rows[state["perm"].long() // state["k"]], state["w"], state["counts"])
    return dict(codes=codes, scale=scale, y=y.to(state["y"].dtype))


# ---------------------------------------------------------------- what a pass cannot do without

def _size(kind):
    return 2 if kind == "f16" else 4


def work(case):
    op = case["op"]
    if op in ("product", "grouped"):
        n = case["n"] if op == "product" else case["T"]
        inn, out, k, E = case["inn"], case["out"], case.get("k", 1), case.get("E", 1)
        used = E * (1 - (1 - k / E) ** n) if op == "grouped" else 1
        return dict(bytes=n * inn * 3 + n * inn / 32 + used * out * inn + n * k * out * _size(case["y"]), flops=2.0 * n * k * inn * out)
    if op == "block":
        T, d, f, E, k = (case[v] for v in ("T", "d", "f", "E", "k"))
        used = E * (1 - (1 - k / E) ** T)
        return dict(bytes=used * 3 * d * f + 4 * T * d + 2 * E * d, flops=6.0 * T * k * d * f + 2.0 * T * E * d)
    T, E, k = case["T"], case["E"], case["k"]
    if op == "loss":
        return dict(bytes=T * (4 * E + 4 * k + (1 if case["padded"] else 0)) + 8 * E, flops=4.0 * T * E)
    d = case["d"]
    return dict(bytes=T * d * (2 + _size(case["dx"])) + T * (8 * E + 8 * k + 1) + 6 * E * d, flops=4.0 * T * d * E + 10.0 * T * E)


# ---------------------------------------------------------------- the definition in 64 bits

def _e4m3(v):
    """Nearest e4m3 value (ties to the even one) of 64-bit values within +-448."""
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    return torch.round(v / step) * step


def _exact_rows(x):
    """Codes and scales of rows; the definition rounds scale, reciprocal and product to 32 bits."""
    n, inn = x.shape
    b = torch.zeros(n, -(-inn // GROUP) * GROUP, dtype=torch.float64, device="cuda")
    b[:, :inn] = x.double()
    b = b.reshape(n, -1, GROUP)
    most = b.abs().max(2, keepdim=True).values
    inverse = torch.where(most > 0, TOP / most, torch.zeros_like(most)).float().double()
    codes = _e4m3((b * inverse).float().double())
    return codes, (most / TOP).float().double()


def _exact_values(x):
    codes, scale = _exact_rows(x)
    return (codes * scale).reshape(x.shape[0], -1)[:, : x.shape[1]]


def _exact_weights(w):
    codes, scale = w
    out, inn = codes.shape
    r = torch.arange(out, device="cuda") // GROUP
    c = torch.arange(inn, device="cuda") // GROUP
    return codes.double() * scale.double()[r][:, c]


def _exact_product(s):
    codes, scale = _exact_rows(s["x"])
    values = (codes * scale).reshape(s["x"].shape[0], -1)[:, : s["inn"]]
    if s["op"] == "product":
        y = values @ _exact_weights(s["w"][0]).t()
    else:
        y, o = torch.empty(s["T"] * s["k"], s["out"], dtype=torch.float64, device="cuda"), s["offsets"].tolist()
        for e in range(s["E"]):
            at = s["perm"][o[e]: o[e + 1]].long() // s["k"]
            if len(at):
                y[o[e]: o[e + 1]] = values[at] @ _exact_weights(s["w"][e]).t()
    return dict(codes=codes.reshape(s["x"].shape[0], -1)[:, : s["inn"]], scale=scale[:, :, 0].t(), y=y)


def _exact_block(s):
    x = s["x"].double()
    logits = x @ s["w_gate"].double().t()
    best, idx = logits.sort(1, descending=True)
    best, idx = best[:, : s["k"]], idx[:, : s["k"]]
    gates = torch.exp(best - best[:, :1])
    gates = gates / gates.sum(1, keepdim=True)
    xq, out = _exact_values(s["x"]), torch.zeros_like(x)
    for e in range(s["E"]):
        t, slot = torch.nonzero(idx == e, as_tuple=True)
        if not len(t):
            continue
        w1, w3, w2 = (_exact_weights(m) for m in s["experts"][e])
        a = xq[t] @ w1.t()
        h = (a * torch.sigmoid(a) * (xq[t] @ w3.t())).half()      # the hidden rows of the framework are fp16
        out[t] += gates[t, slot][:, None] * (_exact_values(h) @ w2.t())
    return dict(out=out)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] in ("product", "grouped"):
        return _exact_product(s)
    if case["op"] == "block":
        return _exact_block(s)
    T, E, k, idx = case["T"], case["E"], case["k"], s["idx"].long()
    keep = torch.ones(T, dtype=torch.bool, device="cuda") if s["valid"] is None else s["valid"] > 0
    z = s["logits"].double()
    p = torch.exp(z - z.max(1, keepdim=True).values)
    p = p / p.sum(1, keepdim=True)
    n = int(keep.sum())
    c = torch.zeros(E, dtype=torch.float64, device="cuda")
    for e in range(E):
        c[e] = ((idx == e).any(1) & keep).sum()
    if case["op"] == "loss":
        mean = p[keep].mean(0)
        counts = torch.cat([c, torch.tensor([float(n)], device="cuda")]).int()
        return dict(counts=counts, mean_prob=mean, loss=(c * mean).sum()[None] * E / (n * k))
    # the loss is E/(n k) sum_e c_e mean_e, its derivative through the softmax; and the softmax over the chosen logits
    dl = torch.zeros(T, E, dtype=torch.float64, device="cuda")
    dp = c[None] * (E / (n * k * n)) * s["d_loss"].double()
    dl += p * (dp - (p * dp).sum(1, keepdim=True))
    a = z.gather(1, idx)
    a = torch.exp(a - a.max(1, keepdim=True).values)
    a = a / a.sum(1, keepdim=True)
    da = s["d_gate"].double()
    da = a * (da - (a * da).sum(1, keepdim=True))
    for j in range(k):
        dl[torch.arange(T, device="cuda"), idx[:, j]] += da[:, j]
    dl[~keep] = 0
    return dict(d_logits=dl, d_x=dl @ s["w_gate"].double(), d_w_gate=dl.t() @ s["x"].double(), d_bias=dl.sum(0))
