"""Balance loss and backward pass of the gate against their formulas in 64 bits and against differences."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24


def gate_layer(E, k, d=64, w_gate=None, bias=None):
    w = torch.zeros(E, d, dtype=torch.float16, device="cuda") if w_gate is None else w_gate
    return mm.Layer(d, 64, k, w, [mm.Expert(mm.PREC_FP16, None, None, None, resident=False) for _ in range(E)], bias)


def softmax(z):
    """Rows of zeros where every entry is -infinity; NaN and +infinity make NaN."""
    with np.errstate(invalid="ignore"):
        m = z.max(1, keepdims=True)
        p = np.exp(z - m)
        p = p / p.sum(1, keepdims=True)
    p[np.all(z == -np.inf, 1)] = 0
    return p


def loss_of(z, idx, valid, E, k):
    keep = valid.astype(bool)
    n = int(keep.sum())
    flat = idx[keep].reshape(-1)
    counts = np.bincount(flat[(flat >= 0) & (flat < E)], minlength=E)
    if n == 0:
        return counts, np.zeros(E), 0.0
    mean = softmax(z[keep]).sum(0) / n
    return counts, mean, E / (n * k) * float(counts @ mean)


def backward_of(z, idx, valid, E, k, counts, d_gate, d_loss):
    T = z.shape[0]
    dl = np.zeros((T, E))
    n = valid.astype(bool).sum()
    if d_loss is not None and n:
        p = softmax(z)
        dl += d_loss * E / (n * k) / n * p * (counts - (p * counts).sum(1, keepdims=True))
    if d_gate is not None:
        for t in range(T):
            ok = (idx[t] >= 0) & (idx[t] < E)
            if not ok.any():
                continue
            g = softmax(z[t][None, idx[t][ok]])[0]
            dg = g * (d_gate[t][ok] - g @ d_gate[t][ok])
            np.add.at(dl[t], idx[t][ok], dg)
    dl[~valid.astype(bool)] = 0
    return dl


def case(rng, T, E, k, padded):
    z = (rng.standard_normal((T, E)) * 1.5).astype(np.float32)
    idx = np.argsort(-z, 1, kind="stable")[:, :k].astype(np.int32)
    valid = (rng.random(T) >= padded).astype(np.uint8)
    return z, idx, valid


def cuda(a, dtype=None):
    return None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda().to(dtype) if dtype else torch.from_numpy(np.ascontiguousarray(a)).cuda()


def run_loss(layer, z, idx, valid, ws=None):
    E = layer.n_experts
    counts = torch.full((E + 1,), -7, dtype=torch.int32, device="cuda")
    mean, loss = torch.full((E,), float("nan"), device="cuda"), torch.full((1,), float("nan"), device="cuda")
    ws = mm.alloc_gate_workspace(layer, z.shape[0]) if ws is None else ws
    mm.moe_balance_loss(layer, z, idx, counts, mean, loss, ws, valid=valid)
    return counts, mean, loss, mm.moe_read_status(ws)


SIZES = [(1, 1, 1), (1, 8, 2), (3, 2, 2), (63, 5, 1), (64, 8, 2), (65, 6, 6), (300, 16, 4), (1000, 32, 8), (2049, 17, 3), (20000, 32, 4), (70001, 8, 2)]


@pytest.mark.parametrize("T,E,k", SIZES)
@pytest.mark.parametrize("padded", [0.0, 0.4, 1.0])
def test_balance_loss(T, E, k, padded):
    print(f"loss T={T} E={E} k={k} padded={padded}", flush=True)
    z, idx, valid = case(np.random.default_rng([T, E, k]), T, E, k, padded)
    counts, mean, loss = loss_of(z.astype(np.float64), idx, valid, E, k)
    zz = z.copy()
    zz[valid == 0] = np.nan                                  # padding is not looked at
    ii = idx.copy()
    ii[valid == 0] = -1
    got_c, got_m, got_l, status = run_loss(gate_layer(E, k), cuda(zz), cuda(ii), None if padded == 0.0 else cuda(valid))
    assert status == 0
    assert got_c.tolist() == counts.tolist() + [int(valid.sum())]
    # a probability: exponentials and their sum of 32 at 2^-22 each, the quotient; then sums of up to T / 2048 + 12 terms in one lane and four wavefronts
    rel = (8 + 64 + T / 2048 + 16) * EPS
    assert np.all(np.abs(got_m.cpu().numpy() - mean) <= mean * rel)
    assert abs(float(got_l) - loss) <= loss * rel
    if T > 1000 and padded == 0.0:
        assert np.linalg.norm(got_m.cpu().numpy() - mean) <= 2.0 ** -21 * np.linalg.norm(mean)


def test_even_load_gives_one():
    E, k, T = 8, 2, 64
    idx = np.stack([np.arange(T) % E, (np.arange(T) + 4) % E], 1).astype(np.int32)
    c, m, l, _ = run_loss(gate_layer(E, k), torch.zeros(T, E, device="cuda"), cuda(idx), None)
    assert c.tolist() == [16] * 8 + [64] and torch.equal(m, torch.full_like(m, 0.125)) and float(l) == 1.0


def test_masked_experts_and_empty_rows():
    """Logits of -infinity, rows that have nothing else, the type's lowest value, and rows with NaN or +infinity."""
    E, k = 6, 2
    z = np.random.default_rng(5).standard_normal((8, E)).astype(np.float32)
    z[1, 2:] = -np.inf
    z[2] = -np.inf
    z[3, :5] = np.finfo(np.float32).min
    z[4] = np.finfo(np.float32).min
    idx = np.argsort(-z, 1, kind="stable")[:, :k].astype(np.int32)
    valid = np.ones(8, np.uint8)
    counts, mean, loss = loss_of(z.astype(np.float64), idx, valid, E, k)
    c, m, l, _ = run_loss(gate_layer(E, k), cuda(z), cuda(idx), None)
    assert c.tolist() == counts.tolist() + [8]
    assert np.all(np.abs(m.cpu().numpy() - mean) <= 100 * EPS * mean) and abs(float(l) - loss) <= 100 * EPS * loss
    dg = np.random.default_rng(6).standard_normal((8, k)).astype(np.float32)
    want = backward_of(z.astype(np.float64), idx, valid, E, k, counts, dg.astype(np.float64), 3.0)
    got = run_backward(gate_layer(E, k), None, z, idx, None, counts, dg, 3.0)["d_logits"]
    assert np.all(np.abs(got - want) <= 2.0 ** -18 * (np.abs(want).max(1, keepdims=True) + 1e-3))
    assert np.all(got[2] == 0)
    for poison in (np.nan, np.inf):
        zz = z.copy()
        zz[6, 3] = poison
        _, m, l, _ = run_loss(gate_layer(E, k), cuda(zz), cuda(idx), None)
        assert bool(m.isnan().all()) and bool(l.isnan().all())
        got = run_backward(gate_layer(E, k), None, zz, idx, None, counts, None, 3.0)["d_logits"]
        assert np.isnan(got[6]).all() and np.isfinite(np.delete(got, 6, 0)).all()
        mask = np.ones(8, np.uint8)
        mask[6] = 0
        _, m, l, _ = run_loss(gate_layer(E, k), cuda(zz), cuda(idx), cuda(mask))
        assert bool(m.isfinite().all()) and bool(l.isfinite().all())


def test_bad_indices_are_reported_and_left_out():
    E, k = 8, 2
    z, idx, valid = case(np.random.default_rng(7), 200, E, k, 0.0)
    idx[3, 0], idx[150, 1] = -1, 8
    counts, mean, loss = loss_of(z.astype(np.float64), idx, valid, E, k)
    c, _, l, status = run_loss(gate_layer(E, k), cuda(z), cuda(idx), None)
    assert status == mm.STATUS_BAD_INDEX and c.tolist() == counts.tolist() + [200] and abs(float(l) - loss) < 1e-5
    dg = np.random.default_rng(8).standard_normal((200, k)).astype(np.float32)
    layer = gate_layer(E, k)
    ws = mm.alloc_gate_workspace(layer, 200)
    dl = torch.full((200, E), float("nan"), device="cuda")
    mm.moe_route_backward(layer, None, cuda(z), cuda(idx), ws, d_gate=cuda(dg), d_logits=dl)
    assert mm.moe_read_status(ws) == mm.STATUS_BAD_INDEX
    want = backward_of(z.astype(np.float64), idx, valid, E, k, counts, dg.astype(np.float64), None)
    assert np.abs(dl.cpu().numpy() - want).max() <= 2.0 ** -18
    mm.moe_route_backward(layer, None, cuda(z), cuda(np.clip(idx, 0, E - 1)), ws, d_gate=cuda(dg), d_logits=dl)
    assert mm.moe_read_status(ws) == 0


# ---------------------------------------------------------------- backward

def run_backward(layer, x, z, idx, valid, counts, dg, d_loss, want=("d_logits",), dx_type=torch.float32, ws=None):
    T, E, d = z.shape[0], layer.n_experts, layer.d_model
    shapes = dict(d_logits=((T, E), torch.float32), d_x=((T, d), dx_type), d_w_gate=((E, d), torch.float32), d_bias=((E,), torch.float32))
    out = {n: torch.full(shapes[n][0], float("nan"), dtype=shapes[n][1], device="cuda") for n in want}
    c = None
    if d_loss is not None:
        n = T if valid is None else int(valid.sum())
        c = cuda(np.concatenate([counts, [n]]).astype(np.int32))
    ws = mm.alloc_gate_workspace(layer, T) if ws is None else ws
    mm.moe_route_backward(layer, cuda(x), cuda(z), cuda(idx), ws, valid=cuda(valid), counts=c, d_gate=cuda(dg),
                          d_loss=None if d_loss is None else torch.full((1,), d_loss, device="cuda"), **out)
    assert mm.moe_read_status(ws) == 0
    return {n: t.cpu().numpy() for n, t in out.items()}


ALL = ("d_logits", "d_x", "d_w_gate", "d_bias")


@pytest.mark.parametrize("T,E,k,d", [(1, 1, 1, 64), (1, 8, 2, 4096), (3, 2, 2, 192), (17, 5, 1, 64), (64, 8, 2, 1024), (130, 6, 6, 320), (333, 16, 4, 832),
                                     (1000, 32, 8, 512), (2049, 17, 3, 128), (4100, 32, 4, 8192), (9000, 8, 2, 2112)])
@pytest.mark.parametrize("padded,half", [(0.0, False), (0.3, True)])
def test_backward(T, E, k, d, padded, half):
    print(f"backward T={T} E={E} k={k} d={d} padded={padded} half={half}", flush=True)
    rng = np.random.default_rng([T, E, k, d])
    z, idx, valid = case(rng, T, E, k, padded)
    x, w = rng.standard_normal((T, d)).astype(np.float16), (rng.standard_normal((E, d)) * 0.05).astype(np.float16)
    dg, d_loss = rng.standard_normal((T, k)).astype(np.float32), 0.5 * T
    counts, _, _ = loss_of(z.astype(np.float64), idx, valid, E, k)
    xs = x.copy()
    xs[valid == 0] = np.nan                                   # padding may hold anything
    zs = z.copy()
    zs[valid == 0] = np.inf
    got = run_backward(gate_layer(E, k, d, cuda(w)), xs, zs, idx, None if padded == 0.0 else valid, counts, dg, d_loss, ALL,
                       torch.float16 if half else torch.float32)
    want = backward_of(z.astype(np.float64), idx, valid, E, k, counts, dg.astype(np.float64), d_loss)
    # d_logits: differences of numbers of the size of d_gate and of the counts, each good to a few 2^-22
    n = max(int(valid.sum()), 1)
    size = np.abs(dg).max(1, keepdims=True) + d_loss * E / (n * k) / n * (counts.max() + 1)
    dl_bound = 64 * 2 * EPS * size * (valid[:, None] > 0)
    assert np.all(np.abs(got["d_logits"] - want) <= dl_bound)
    wf, xf = w.astype(np.float64), x.astype(np.float64)
    # a sum of E (T) terms in 32 bits on top of the terms' own bounds; the split of a term in two halves of 11 bits is good to 2^-21
    dx_bound = dl_bound * np.abs(wf).sum(0) + (np.abs(want) @ np.abs(wf)) * (E + 16) * EPS
    ref = want @ wf
    if half:
        dx_bound = dx_bound + np.abs(ref) * 2.0 ** -11 + 2.0 ** -25
    assert np.all(np.abs(got["d_x"].astype(np.float64) - ref) <= dx_bound)
    xv = xf * (valid[:, None] > 0)
    mag = np.abs(want).T @ np.abs(xv)
    dw_bound = dl_bound.T @ np.abs(xv) + mag * (T / 8 + 32) * EPS            # (dl_bound is the same for all experts)
    err = np.abs(got["d_w_gate"] - want.T @ xv)
    assert np.all(err <= dw_bound)
    assert np.linalg.norm(err) <= 2.0 ** -18 * np.linalg.norm(want.T @ xv) + 2.0 ** -30 * np.linalg.norm(mag)
    db_bound = np.broadcast_to(dl_bound, want.shape).sum(0) + np.abs(want).sum(0) * (T / 2048 + 32) * EPS
    assert np.all(np.abs(got["d_bias"] - want.sum(0)) <= db_bound)


@pytest.mark.parametrize("want", [("d_logits",), ("d_x",), ("d_w_gate",), ("d_bias",), ("d_x", "d_bias")])
def test_each_gradient_alone(want):
    T, E, k, d = 200, 8, 2, 256
    rng = np.random.default_rng(9)
    z, idx, valid = case(rng, T, E, k, 0.2)
    x, w = rng.standard_normal((T, d)).astype(np.float16), rng.standard_normal((E, d)).astype(np.float16)
    dg = rng.standard_normal((T, k)).astype(np.float32)
    counts, _, _ = loss_of(z.astype(np.float64), idx, valid, E, k)
    layer = gate_layer(E, k, d, cuda(w))
    whole = run_backward(layer, x, z, idx, valid, counts, dg, 7.0, ALL)
    one = run_backward(layer, x if "d_w_gate" in want else None, z, idx, valid, counts, dg, 7.0, want)
    for n in want:
        assert np.array_equal(one[n], whole[n]), n
    # the two sources add up
    a, b = (run_backward(layer, x, z, idx, valid, counts, g, l, ALL) for g, l in ((dg, None), (None, 7.0)))
    for n in ALL:
        assert np.allclose(a[n] + b[n], whole[n], rtol=1e-4, atol=1e-4 * np.abs(whole[n]).max()), n


def test_an_expert_chosen_twice():
    """Its two gates are two terms of the softmax over the chosen logits."""
    E, k, T = 4, 3, 5
    rng = np.random.default_rng(10)
    z = rng.standard_normal((T, E)).astype(np.float32)
    idx = np.array([[0, 0, 1], [2, 2, 2], [3, 1, 3], [0, 1, 2], [1, 1, 0]], np.int32)
    dg = rng.standard_normal((T, k)).astype(np.float32)
    got = run_backward(gate_layer(E, k), None, z, idx, None, None, dg, None)["d_logits"]
    want = backward_of(z.astype(np.float64), idx, np.ones(T), E, k, None, dg.astype(np.float64), None)
    assert np.all(np.abs(got - want) <= 64 * 2 * EPS * np.abs(dg).max(1, keepdims=True))


def test_against_differences():
    """Of f(x, W, b) = sum(d_gate * gates) + 3 loss with the counts and the choice held, through the 64-bit formulas forward."""
    T, E, k, d = 24, 6, 2, 64
    rng = np.random.default_rng(11)
    x, w = rng.standard_normal((T, d)).astype(np.float16), (rng.standard_normal((E, d)) * 0.2).astype(np.float16)
    b, dg = rng.standard_normal(E).astype(np.float32), rng.standard_normal((T, k)).astype(np.float32)
    layer = gate_layer(E, k, d, cuda(w), cuda(b))
    logits, idx, gate = torch.empty(T, E, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda"), torch.empty(T, k, device="cuda")
    mm.moe_route_logits(layer, cuda(x), logits, idx, gate)
    other_idx, other_gate = torch.empty_like(idx), torch.empty_like(gate)
    mm.moe_route(layer, cuda(x), other_idx, other_gate)
    assert torch.equal(idx, other_idx) and torch.equal(gate, other_gate)
    z, idx = logits.cpu().numpy(), idx.cpu().numpy()
    xf, wf, bf = x.astype(np.float64), w.astype(np.float64), b.astype(np.float64)
    assert np.abs(z - (xf @ wf.T + bf)).max() <= 1e-4
    valid = np.ones(T, np.uint8)
    counts, _, _ = loss_of(z, idx, valid, E, k)
    got = run_backward(layer, x, z, idx, None, counts, dg, 3.0, ALL)

    def f(xf, wf, bf):
        z = xf @ wf.T + bf
        gates = softmax(np.take_along_axis(z, idx.astype(np.int64), 1))
        return (gates * dg).sum() + 3.0 * E / (T * k) * float(counts @ softmax(z).mean(0))

    h = 1e-5
    for _ in range(24):
        t, e, c = rng.integers(T), rng.integers(E), rng.integers(d)
        for name, at, args in (("d_x", (t, c), 0), ("d_w_gate", (e, c), 1), ("d_bias", (e,), 2)):
            lo, hi = [xf, wf, bf], [xf, wf, bf]
            lo[args], hi[args] = lo[args].copy(), hi[args].copy()
            lo[args][at] -= h
            hi[args][at] += h
            diff = (f(*hi) - f(*lo)) / (2 * h)
            assert abs(diff - got[name][at]) <= 1e-4 * max(1.0, abs(diff)), (name, at)


def test_same_bits_again_in_a_graph_and_on_another_stream():
    T, E, k, d = 1500, 32, 4, 512
    rng = np.random.default_rng(12)
    w = (rng.standard_normal((E, d)) * 0.05).astype(np.float16)
    layer = gate_layer(E, k, d, cuda(w))
    new = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    x, logits, idx, gate = new(T, d, t=torch.float16), new(T, E), new(T, k, t=torch.int32), new(T, k)
    counts, mean, loss, one = new(E + 1, t=torch.int32), new(E), new(1), torch.full((1,), 2.0, device="cuda")
    dg, valid = cuda(rng.standard_normal((T, k)).astype(np.float32)), cuda((rng.random(T) > 0.2).astype(np.uint8))
    res = [new(T, E), new(T, d), new(E, d), new(E)]
    ws = mm.alloc_gate_workspace(layer, T)

    def step():
        mm.moe_route_logits(layer, x, logits, idx, gate)
        mm.moe_balance_loss(layer, logits, idx, counts, mean, loss, ws, valid=valid)
        mm.moe_route_backward(layer, x, logits, idx, ws, valid=valid, counts=counts, d_gate=dg, d_loss=one, d_logits=res[0], d_x=res[1],
                              d_w_gate=res[2], d_bias=res[3])

    x.copy_(cuda(rng.standard_normal((T, d)).astype(np.float16)))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        x.copy_(cuda(rng.standard_normal((T, d)).astype(np.float16)))
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (counts, mean, loss, *res)]
        for t in res:
            t.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        for a, b in zip(got, (counts, mean, loss, *res)):
            assert torch.equal(a, b), i


def test_tokens_off_16_byte_boundaries():
    T, E, k, d = 40, 8, 2, 128
    rng = np.random.default_rng(13)
    z, idx, valid = case(rng, T, E, k, 0.0)
    flat = rng.standard_normal(T * d + 5).astype(np.float16)
    layer, dg = gate_layer(E, k, d), rng.standard_normal((T, k)).astype(np.float32)
    res = []
    for x in (cuda(flat)[5:].view(T, d), cuda(flat[5:]).view(T, d)):
        dw, dx = torch.empty(E, d, device="cuda"), torch.empty(T * d + 1, dtype=torch.float16, device="cuda")[1:].view(T, d)
        mm.moe_route_backward(layer, x, cuda(z), cuda(idx), mm.alloc_gate_workspace(layer, T), d_gate=cuda(dg), d_w_gate=dw, d_x=dx)
        res.append((dw, dx))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])


def test_binding_refuses_what_does_not_fit():
    T, E, k = 10, 8, 2
    layer = gate_layer(E, k)
    z, idx = torch.zeros(T, E, device="cuda"), torch.zeros(T, k, dtype=torch.int32, device="cuda")
    c, m, l, ws = torch.zeros(E + 1, dtype=torch.int32, device="cuda"), torch.zeros(E, device="cuda"), torch.zeros(1, device="cuda"), mm.alloc_gate_workspace(layer, T)
    mm.moe_balance_loss(layer, z, idx, c, m, l, ws)
    for bad in (dict(z=z[:, :7]), dict(z=torch.zeros(T, E + 8, device="cuda")[:, :E]), dict(z=z.double()), dict(idx=idx.long()), dict(idx=idx[:9]),
                dict(c=c[:E]), dict(m=m.cpu()), dict(ws=ws[256:]), dict(ws=None), dict(valid=torch.zeros(T, device="cuda"))):
        a = dict(z=z, idx=idx, c=c, m=m, ws=ws, valid=None) | bad
        with pytest.raises(mm.MoeError):
            mm.moe_balance_loss(layer, a["z"], a["idx"], a["c"], a["m"], l, a["ws"], valid=a["valid"])
    with pytest.raises(mm.MoeError):
        mm.moe_route_backward(layer, None, z, idx, ws, d_gate=torch.zeros(T, k, device="cuda"), d_x=torch.zeros(T, 64, dtype=torch.bfloat16, device="cuda"))
    other = torch.cuda.current_device()
    assert z.get_device() == other
