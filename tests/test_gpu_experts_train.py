"""Forward and backward pass of 16-bit experts against their formulas in 64 bits and against differences."""
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm
from tests.train_ref import Ref, assert_within

pytestmark = pytest.mark.gpu


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).half()


class Block:
    """Seeded weights, tokens and a grouping: idx [T,k], -1 for a pair in no group."""

    def __init__(self, seed, T, d, f, E, k, idx=None, sigma=None, rest=7.0):
        g = gen(seed)
        self.T, self.d, self.f, self.E, self.k = T, d, f, E, k
        s1, s2 = (d ** -0.5, f ** -0.5) if sigma is None else (sigma, sigma)
        self.w1, self.w3, self.w2 = normal(g, E, f, d, scale=s1), normal(g, E, f, d, scale=s1), normal(g, E, d, f, scale=s2)
        self.x, self.d_out = normal(g, T, d), normal(g, T, d, scale=0.5)
        taste = torch.rand(T, E, generator=g, device="cuda")
        self.idx = taste.topk(k, 1).indices.int() if idx is None else idx.int()
        self.gate = torch.rand(T, k, generator=g, device="cuda") + 0.1
        self.group()
        self.layer = mm.Layer(d, f, k, torch.zeros(E, d, dtype=torch.float16, device="cuda"),
                              [mm.Expert(mm.PREC_FP16, mm.Mat(self.w1[e]), mm.Mat(self.w3[e]), mm.Mat(self.w2[e])) for e in range(E)])
        self.ws = mm.alloc_experts_workspace(self.layer, T)
        self.a, self.u = (torch.full((T * k, f), rest, dtype=torch.float16, device="cuda") for _ in range(2))
        self.out = torch.full((T, d), rest, dtype=torch.float16, device="cuda")

    def group(self):
        flat = self.idx.reshape(-1).long()
        key = torch.where(flat < 0, self.E, flat)
        self.perm = torch.sort(key, stable=True).indices.int()
        counts = torch.bincount(key, minlength=self.E + 1)[: self.E]
        self.offsets = torch.nn.functional.pad(counts.cumsum(0), (1, 0)).int()
        self.counts = counts.tolist()
        self.n = sum(self.counts)

    def ref(self):
        groups = list(self.perm[: self.n].long().split(self.counts))
        return Ref(self.x, self.w1, self.w3, self.w2, groups, self.gate.double().reshape(-1), self.k)

    def forward(self, **more):
        args = dict(gate=self.gate, offsets=self.offsets, perm=self.perm) | more
        mm.moe_experts_forward(self.layer, self.x, args["gate"], args["offsets"], args["perm"], self.a, self.u, self.out, self.ws)

    def grads(self, dtype=torch.float32, fill=9.0):
        new = lambda *s, t=dtype: torch.full(s, fill, dtype=t, device="cuda")  # noqa: E731
        self.d_x, self.d_gate = new(self.T, self.d), new(self.T, self.k, t=torch.float32)
        self.g1, self.g3, self.g2 = new(self.E, self.f, self.d), new(self.E, self.f, self.d), new(self.E, self.d, self.f)
        self.d_w = mm.ExpertGrads([(self.g1[e], self.g3[e], self.g2[e]) for e in range(self.E)])

    def backward(self, accumulate=False, **more):
        args = dict(gate=self.gate, offsets=self.offsets, perm=self.perm, d_x=self.d_x, d_gate=self.d_gate, d_w=self.d_w) | more
        mm.moe_experts_backward(self.layer, self.x, args["gate"], args["offsets"], args["perm"], self.a, self.u, self.d_out, self.ws,
                                d_x=args["d_x"], d_gate=args["d_gate"], d_w=args["d_w"], accumulate=accumulate)

    def results(self):
        return [t.clone() for t in (self.d_x, self.d_gate, self.g1, self.g3, self.g2)]

    def check_forward(self):
        (a, ea), (u, eu), (out, eo) = self.ref().forward()
        assert_within(self.a[: self.n], a, ea, "a")
        assert_within(self.u[: self.n], u, eu, "u")
        assert_within(self.out, out, eo, "out")

    def check_backward(self, before=None):
        half = self.d_x.dtype == torch.float16
        r = self.ref().backward(self.a, self.u, self.d_out)
        assert_within(self.d_gate, r["d_gate"][0], r["d_gate"][1], "d_gate")
        assert_within(self.d_x, *r["d_x"], "d_x", half)
        for name, got in (("w1", self.g1), ("w3", self.g3), ("w2", self.g2)):
            for e, (v, b) in enumerate(r[name]):
                more = 0.0 if before is None else before
                assert_within(got[e], v + more, b + 2.0 ** -23 * (abs(more) + v.abs()), f"{name} of expert {e}", half)


SHAPES = [(1, 64, 64, 1, 1), (1, 128, 192, 4, 2), (2, 256, 512, 4, 2), (16, 256, 512, 4, 2), (33, 192, 320, 5, 2), (77, 512, 64, 3, 1), (300, 128, 704, 2, 2),
          (513, 64, 192, 1, 1), (257, 320, 256, 8, 8), (600, 320, 448, 2, 1), (1000, 1024, 320, 8, 2), (90, 2048, 128, 32, 8), (19, 8192, 128, 2, 1), (19, 128, 16384, 2, 2)]


@pytest.mark.parametrize("T,d,f,E,k", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_forward_and_backward(T, d, f, E, k, dtype):
    b = Block(T + d + f, T, d, f, E, k)
    b.forward()
    b.check_forward()
    b.grads(dtype)
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("rows", [1, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 95, 96, 97, 127, 128, 129, 160, 191, 192, 193, 224, 255, 256, 257, 320, 385])
def test_numbers_of_rows(rows):
    """One expert with so many rows beside one with three and one with none."""
    idx = torch.cat([torch.full((rows,), 1), torch.full((3,), 2)]).reshape(-1, 1).cuda()
    idx = idx[torch.randperm(rows + 3, generator=torch.Generator().manual_seed(rows)).cuda()]
    b = Block(rows, rows + 3, 128, 320, 4, 1, idx=idx)
    b.forward()
    b.check_forward()
    b.grads()
    b.backward()
    b.check_backward()
    for g in (b.g1, b.g3, b.g2):
        assert float(g[0].abs().max()) == 0 and float(g[3].abs().max()) == 0


def test_training_batch():
    b = Block(3, 2500, 1024, 1408, 8, 2)
    b.forward()
    b.check_forward()
    b.grads(torch.float16)
    b.backward()
    b.check_backward()


def test_padding_holds_anything():
    T, k = 200, 2
    g = gen(5)
    idx = torch.rand(T, 4, generator=g, device="cuda").topk(k, 1).indices
    gone = torch.rand(T, generator=g, device="cuda") < 0.3
    idx[gone] = -1
    idx[7] = torch.tensor([-1, 2], device="cuda")           # one pair of two
    gone[7] = False
    b = Block(5, T, 192, 256, 4, k, idx=idx)
    clean = b.x.clone(), b.d_out.clone()
    b.x[gone], b.d_out[gone], b.gate[gone] = float("nan"), float("inf"), float("nan")
    b.forward()
    b.grads()
    b.backward()
    for t in (b.out, b.d_x, b.d_gate):
        assert float(t[gone].abs().max()) == 0
    assert (b.a[b.n:] == 7).all() and (b.u[b.n:] == 7).all()
    b.x, b.d_out = clean
    b.gate[gone] = 0
    b.check_forward()
    b.check_backward()


def test_no_rows_at_all():
    b = Block(1, 5, 64, 64, 2, 1, idx=torch.full((5, 1), -1).cuda())
    b.forward()
    b.grads()
    b.backward()
    for t in (b.out, b.d_x, b.d_gate, b.g1, b.g3, b.g2):
        assert float(t.abs().max()) == 0
    b.grads()
    b.backward(accumulate=True)
    assert (b.g1 == 9).all() and (b.g3 == 9).all() and (b.g2 == 9).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_accumulate(dtype):
    b = Block(11, 150, 192, 320, 3, 2)
    b.forward()
    b.grads(dtype, fill=0.25)
    b.backward(accumulate=True)
    b.check_backward(before=0.25)


def test_each_gradient_alone_has_the_same_bits():
    b = Block(12, 130, 128, 192, 4, 2)
    b.forward()
    b.grads()
    b.backward()
    every = b.results()
    none = dict(d_x=None, d_gate=None, d_w=None)
    b.grads()
    b.backward(**none | dict(d_x=b.d_x))
    assert torch.equal(b.d_x, every[0]) and (b.g1 == 9).all() and (b.d_gate == 9).all()
    b.grads()
    b.backward(**none | dict(d_gate=b.d_gate))
    assert torch.equal(b.d_gate, every[1]) and (b.d_x == 9).all()
    b.grads()
    b.backward(**none | dict(d_w=mm.ExpertGrads([(None, b.g3[0], None), None, (b.g1[2], None, b.g2[2]), (None, None, None)])))
    assert torch.equal(b.g3[0], every[3][0]) and torch.equal(b.g1[2], every[2][2]) and torch.equal(b.g2[2], every[4][2])
    assert (b.g3[1:] == 9).all() and (b.g1[:2] == 9).all() and (b.g1[3] == 9).all() and (b.g2[:2] == 9).all() and (b.d_x == 9).all()


@pytest.mark.parametrize("T", [1, 70, 500])
def test_one_expert_without_a_grouping(T):
    """A dense gated block: no offsets, no perm, no gates."""
    b = Block(T, T, 192, 448, 1, 1)
    b.gate.fill_(1.0)
    b.perm = torch.arange(T, device="cuda", dtype=torch.int32)
    b.forward()
    kept = b.out.clone()
    b.grads()
    b.backward()
    every = b.results()
    b.out.zero_()
    b.forward(gate=None, offsets=None, perm=None)
    assert torch.equal(b.out, kept)
    b.check_forward()
    b.grads()
    b.backward(gate=None, offsets=None, perm=None)
    assert all(torch.equal(p, q) for p, q in zip(b.results(), every))
    b.check_backward()


def test_pairs_in_grouped_order_without_perm():
    idx = torch.tensor([0] * 40 + [1] * 30 + [2] * 5).reshape(-1, 1).cuda()
    b = Block(2, 75, 64, 128, 3, 1, idx=idx)
    b.forward()
    kept = b.out.clone()
    b.forward(perm=None)
    assert torch.equal(b.out, kept)


def test_the_block_that_inference_computes():
    """Gating, grouping and experts by the calls of a training program, beside moe_layer_forward."""
    T, d, f, E, k = 300, 256, 512, 4, 2
    b = Block(21, T, d, f, E, k)
    b.layer = mm.Layer(d, f, k, normal(gen(4), E, d, scale=0.05), b.layer.experts)
    ws = mm.alloc_workspace(b.layer, T)
    out = torch.empty_like(b.out)
    mm.moe_layer_forward(b.layer, b.x, out, ws)
    logits, idx = torch.empty(T, E, device="cuda"), torch.empty(T, k, dtype=torch.int32, device="cuda")
    mm.moe_route_logits(b.layer, b.x, logits, idx, b.gate)
    counts, offsets, perm = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (E, E + 1, T * k))
    mm.moe_permute(b.layer, idx, counts, offsets, perm, ws)
    mm.moe_experts_forward(b.layer, b.x, b.gate, offsets, perm, b.a, b.u, b.out, b.ws)
    b.idx = idx
    b.group()
    assert torch.equal(b.perm, perm)
    b.check_forward()
    # both round hidden rows and outputs to fp16: two roundings each, in other places of the sums
    assert float((out.double() - b.out.double()).norm() / b.out.double().norm()) <= 2e-3


def test_graph_replays_other_stream_and_shared_workspace():
    b, c = Block(31, 180, 128, 320, 4, 2), Block(32, 64, 128, 320, 4, 2)
    c.ws = b.ws
    want = []
    for v in (b, c):
        v.forward()
        v.grads()
        v.backward()
        want.append([v.a.clone(), v.u.clone(), v.out.clone()] + v.results())
    torch.cuda.synchronize()
    graphs, stream = [], torch.cuda.Stream()
    for v in (b, c):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=stream):
            v.forward()
            v.backward()
        graphs.append(g)
    for turn in range(3):
        for v in (b, c):
            for t in (v.a, v.u, v.out, v.d_x, v.d_gate, v.g1, v.g3, v.g2):
                t.fill_(3 + turn)
        b.ws.random_(0, 255)                                   # a workspace carries nothing over
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for v, w in zip((b, c), want):
            assert all(torch.equal(p, q) for p, q in zip([v.a, v.u, v.out] + v.results(), w))
        b.x.sum().item()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.out.zero_()
        b.forward()
        b.backward()
    side.synchronize()
    assert all(torch.equal(p, q) for p, q in zip([b.a, b.u, b.out] + b.results(), want[0]))


def test_groupings_that_are_none():
    """Offsets and perm that no moe_permute gives: nothing outside the arrays is touched, what lies in a group and names a pair is computed."""
    T, d, f, E, k = 60, 64, 128, 4, 2
    b = Block(8, T, d, f, E, k)
    big = torch.full((T * k + 256, f), 5.0, dtype=torch.float16, device="cuda")
    b.a = big[128: 128 + T * k]
    for offsets, perm in (([-7, 200, 50, 1000, 2 ** 31 - 1], b.perm), ([0, 90, 30, 20, 10], b.perm), ([5, 5, 5, 5, 5], b.perm),
                          (b.offsets.tolist(), torch.randint(-(2 ** 31), 2 ** 31 - 1, (T * k,), device="cuda", dtype=torch.int32)),
                          (b.offsets.tolist(), torch.zeros(T * k, dtype=torch.int32, device="cuda"))):
        o = torch.tensor(offsets, dtype=torch.int32, device="cuda")
        b.forward(offsets=o, perm=perm)
        b.grads()
        b.backward(offsets=o, perm=perm)
        torch.cuda.synchronize()
        assert (big[:128] == 5).all() and (big[128 + T * k:] == 5).all()


def test_large_values_and_infinities():
    """Gradients past the range of fp16 on the way are infinities or NaN in what they reach and nowhere else."""
    b = Block(9, 40, 64, 128, 2, 1, idx=torch.tensor([0, 1] * 20).reshape(-1, 1).cuda())
    b.forward()
    b.d_out[0, 3] = float("inf")                               # a row of expert 0
    b.grads()
    b.backward()
    assert not torch.isfinite(b.g1[0]).all() and torch.isfinite(b.g1[1]).all() and torch.isfinite(b.g2[1]).all()
    assert not torch.isfinite(b.d_gate[0]).all() and torch.isfinite(b.d_gate[1:]).all() and torch.isfinite(b.d_x[1:]).all()
    b.d_out[0, 3] = 0
    b.a[0], b.a[1] = 60000.0, -60000.0                         # silu saturates
    b.backward()
    assert torch.isfinite(b.d_x).all()
    r = b.ref().backward(b.a, b.u, b.d_out)
    assert_within(b.d_gate, *r["d_gate"], "d_gate")
    assert_within(b.d_x, *r["d_x"], "d_x")
    for e in range(2):
        assert_within(b.g1[e], *r["w1"][e], "w1")
        assert_within(b.g3[e], *r["w3"][e], "w3")
        # silu(60000) u g passes 65504, the largest fp16, wherever |u g| > 1.0918: those hidden values are infinities, and with them their columns of d_w2
        past = (60000.0 * b.u[0].double() * b.gate[0, 0].double()).abs() > 65520 if e == 0 else torch.zeros(128, dtype=torch.bool, device="cuda")
        assert not torch.isfinite(b.g2[e][:, past]).any() and past.any() == (e == 0)
        assert_within(b.g2[e][:, ~past], *(v[:, ~past] for v in r["w2"][e]), "w2")


@pytest.mark.parametrize("what", ["x", "gate", "w1", "w3", "w2"])
def test_against_differences(what):
    """The derivative of sum(out * d_out) in 64 bits along a direction, from differences; the kernels' gradients are off by their roundings, 2e-3 of |gradient| |direction|."""
    b = Block(41, 50, 64, 128, 3, 2)
    b.forward()
    b.grads()
    b.backward()
    grad = dict(x=b.d_x, gate=b.d_gate, w1=b.g1, w3=b.g3, w2=b.g2)[what].double()
    way = torch.randn(grad.shape, generator=gen(6), device="cuda", dtype=torch.float64)

    def loss(step):
        r = b.ref()
        if what == "x":
            r.x = r.x + step * way
        elif what == "gate":
            r.g = r.g + step * way.reshape(-1)
        else:
            i = ("w1", "w3", "w2").index(what)
            r.w = [tuple(m + step * way[e] if j == i else m for j, m in enumerate(w)) for e, w in enumerate(r.w)]
        return float((r.forward()[2][0] * b.d_out.double()).sum())

    step = 1e-5
    slope = (loss(step) - loss(-step)) / (2 * step)
    assert abs(slope - float((grad * way).sum())) <= 2e-3 * float(grad.norm()) * float(way.norm())


def test_a_step_of_training():
    """Gate, grouping, experts, balance loss, both backward passes and clipping, as a program runs them, beside derivatives by torch in 64 bits."""
    T, d, f, E, k, scale = 120, 128, 192, 4, 2, 256.0
    b = Block(51, T, d, f, E, k)
    w_gate = normal(gen(7), E, d, scale=0.3)
    layer = mm.Layer(d, f, k, w_gate, b.layer.experts)
    new = lambda *s, t=torch.float32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    logits, idx, gate = new(T, E), new(T, k, t=torch.int32), new(T, k)
    counts, offsets, perm = new(E, t=torch.int32), new(E + 1, t=torch.int32), new(T * k, t=torch.int32)
    ws, gate_ws, train_ws = mm.alloc_workspace(layer, T), mm.alloc_gate_workspace(layer, T), mm.alloc_experts_workspace(layer, T)
    mm.moe_route_logits(layer, b.x, logits, idx, gate)
    mm.moe_permute(layer, idx, counts, offsets, perm, ws)
    mm.moe_experts_forward(layer, b.x, gate, offsets, perm, b.a, b.u, b.out, train_ws)
    loss_counts, mean_prob, loss = new(E + 1, t=torch.int32), new(E), new(1)
    mm.moe_balance_loss(layer, logits, idx, loss_counts, mean_prob, loss, gate_ws)
    d_out = (b.d_out.float() * scale / 64).half()
    b.grads()
    mm.moe_experts_backward(layer, b.x, gate, offsets, perm, b.a, b.u, d_out, train_ws, d_x=b.d_x, d_gate=b.d_gate, d_w=b.d_w)
    d_loss, d_xg, d_wg, d_logits = torch.full((1,), scale, device="cuda"), new(T, d), new(E, d), new(T, E)
    mm.moe_route_backward(layer, b.x, logits, idx, gate_ws, counts=loss_counts, d_gate=b.d_gate, d_loss=d_loss, d_logits=d_logits, d_x=d_xg, d_w_gate=d_wg)
    grads = [b.g1, b.g3, b.g2, d_wg]
    before = [g.clone() for g in grads]
    norm = new(1)
    mm.moe_clip_gradients(mm.GradList(grads), 0.01, norm, mm.alloc_clip_workspace(4), unscale=1 / scale)

    x, wg = b.x.double().requires_grad_(), w_gate.double().requires_grad_()
    w = [t.double().requires_grad_() for t in (b.w1, b.w3, b.w2)]
    z = x @ wg.t()
    g = torch.softmax(z.gather(1, idx.long()), 1)
    out = torch.zeros_like(x)
    for e in range(E):
        t, s = torch.nonzero(idx == e, as_tuple=True)
        a, u = x[t] @ w[0][e].t(), x[t] @ w[1][e].t()
        out = out.index_add(0, t, g[t, s][:, None] * ((torch.nn.functional.silu(a) * u) @ w[2][e].t()))
    c = loss_counts[:E].double()
    total = (out * d_out.double()).sum() + scale * E / (T * k) * (c * torch.softmax(z, 1).mean(0)).sum()
    total.backward()
    near = lambda p, q: float((p.double() - q).norm() / q.norm())  # noqa: E731
    assert near(b.out, out.detach()) <= 2e-3
    for got, want in zip(before[:3], w):
        assert near(got, want.grad) <= 2e-3
    # through d_gate, 32 bits from rows rounded to fp16
    assert near(d_wg * 0 + before[3], wg.grad) <= 4e-3 and near(b.d_x.double() + d_xg.double(), x.grad) <= 4e-3
    length = sum(float(p.double().square().sum()) for p in before) ** 0.5 / scale
    assert abs(float(norm) - length) <= 2.0 ** -23 * length and length > 0.01
    factor = 0.01 / (length + 1e-6) / scale
    for p, q in zip(before, grads):
        assert float((q.double() - p.double() * factor).abs().max()) <= 2.0 ** -22 * float(p.abs().max()) * factor


def test_tokens_are_not_taken_for_others():
    """Distinct tokens in many chunks: every row of out is its own token's."""
    T = 3000
    b = Block(61, T, 64, 64, 2, 1, idx=(torch.arange(T) % 2).reshape(-1, 1).cuda())
    b.x.copy_(((torch.arange(T, device="cuda") % 13 + 1) / 8).half()[:, None].expand(T, 64))
    b.forward()
    b.check_forward()


def test_in_place():
    """out may take the place of x, d_x the place of d_out."""
    b = Block(71, 90, 128, 192, 3, 2)
    b.forward()
    b.grads(torch.float16)
    b.backward()
    out, d_x = b.out.clone(), b.d_x.clone()
    x = b.x.clone()
    mm.moe_experts_forward(b.layer, x, b.gate, b.offsets, b.perm, b.a, b.u, x, b.ws)
    assert torch.equal(x, out)
    d = b.d_out.clone()
    mm.moe_experts_backward(b.layer, b.x, b.gate, b.offsets, b.perm, b.a, b.u, d, b.ws, d_x=d)
    assert torch.equal(d, d_x)


def test_workspaces_of_other_sizes():
    """Room for fewer partial results, for none, and what more tokens ask for."""
    T, d, f, E, k = 16, 256, 512, 4, 2
    b = Block(81, T, d, f, E, k)
    one, full = T * k * d * 4, b.ws.numel()                   # a set of rows; as many as 16 lie at the end of a workspace
    for n in (full, full - 256, full - 6 * one, full - 15 * one, mm.experts_workspace_bytes(b.layer, 900)):
        b.ws = torch.empty(n, dtype=torch.uint8, device="cuda")
        for t in (b.a, b.u, b.out):
            t.fill_(7.0)
        b.forward()
        b.check_forward()
        b.grads()
        b.backward()
        b.check_backward()
    b.ws = torch.empty(full - 15 * one - 256, dtype=torch.uint8, device="cuda")
    for call in (b.forward, b.backward):
        with pytest.raises(mm.MoeError) as e:
            call()
        assert e.value.code == mm.MOE_EWORKSPACE


@pytest.mark.parametrize("counts", [(2600, 300, 9, 0, 91), (1, 2304, 1, 257, 513), (40, 40, 40, 40, 2048 + 33), (0, 0, 3000, 0, 0)])
@pytest.mark.parametrize("d,f", [(192, 704), (1344, 128)])
def test_loads_of_all_kinds(counts, d, f):
    """Experts of more chunks than go side by side, beside small ones and none."""
    idx = torch.cat([torch.full((n,), e) for e, n in enumerate(counts)])
    idx = idx[torch.randperm(len(idx), generator=torch.Generator().manual_seed(d))].reshape(-1, 1).cuda()
    b = Block(d + counts[0], len(idx), d, f, 5, 1, idx=idx)
    b.forward()
    b.check_forward()
    b.grads(torch.float16)
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("T,d,f", [(262143, 8192, 64), (140000, 64, 16384)])
def test_offsets_past_32_bits(T, d, f):
    """The last hundred tokens are an expert's of their own: their rows, their gradients and the expert's."""
    n = 100
    idx = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    idx[-n:] = 1
    b = Block(83, T, d, f, 2, 1, idx=idx)
    b.forward()
    b.grads()
    b.backward()
    ref = Ref(b.x[-n:], b.w1[1:], b.w3[1:], b.w2[1:], [torch.arange(n, device="cuda")], b.gate[-n:].double().reshape(-1), 1)
    for got, (v, bound), what in zip((b.a, b.u, b.out), ref.forward(), ("a", "u", "out")):
        assert_within(got[-n:], v, bound, what)
    r = ref.backward(b.a[-n:], b.u[-n:], b.d_out[-n:])
    assert_within(b.d_gate[-n:], *r["d_gate"], "d_gate")
    assert_within(b.d_x[-n:], *r["d_x"], "d_x")
    for name, got in (("w1", b.g1), ("w3", b.g3), ("w2", b.g2)):
        assert_within(got[1], *r[name][0], name)


@pytest.mark.parametrize("counts", [(2600, 300, 9, 0, 91), (1, 2304, 1, 257, 513), (640, 576, 513, 600, 703), (3000, 1, 0, 0, 0)])
@pytest.mark.parametrize("dtype,accumulate", [(torch.float32, False), (torch.float16, True)])
def test_large_tiles(counts, dtype, accumulate):
    """Matrices so large and experts with so many rows that the gradients of matrices are made of tiles of 256 x 256, whose last ones are cut off."""
    idx = torch.cat([torch.full((n,), e) for e, n in enumerate(counts)])
    idx = idx[torch.randperm(len(idx), generator=torch.Generator().manual_seed(counts[1]))].reshape(-1, 1).cuda()
    b = Block(counts[0], len(idx), 1472, 2368, 5, 1, idx=idx)
    b.forward()
    b.check_forward()
    b.grads(dtype, fill=0.25)
    b.backward(accumulate=accumulate)
    b.check_backward(before=0.25 if accumulate else None)


@pytest.mark.parametrize("rows", [1, 31, 32, 33, 63, 64, 65, 128, 129, 200])
@pytest.mark.parametrize("d,f", [(1088, 1984), (64, 64)])
def test_small_tiles(rows, d, f):
    """Rows of one expert beside one with three and one with none, in one tile after the other of 128 x 128."""
    idx = torch.cat([torch.full((rows,), 7), torch.full((3,), 2)]).reshape(-1, 1).cuda()
    b = Block(rows, rows + 3, d, f, 16, 1, idx=idx)
    b.forward()
    b.grads(torch.float16)
    b.backward()
    b.check_backward()
    before = b.results()
    b.backward(accumulate=True)
    b.g1, b.g3, b.g2 = b.g1 / 2, b.g3 / 2, b.g2 / 2           # twice the same, rounded once more
    for got, want in zip((b.g1, b.g3, b.g2), before[2:]):
        assert float((got.double() - want.double()).abs().max()) <= 2.0 ** -10 * float(want.abs().max())


@pytest.mark.parametrize("T,k", [(1, 2), (40, 2), (700, 4)])
def test_matrices_larger_than_the_last_level_cache(T, k):
    """277 MB of them; experts of up to 128 rows and of more, some split."""
    idx = torch.rand(T, 16, generator=gen(T), device="cuda").mul(torch.linspace(0.2, 1, 16, device="cuda")).topk(k, 1).indices
    b = Block(91 + T, T, 1024, 2816, 16, k, idx=idx)
    b.forward()
    b.check_forward()
    b.grads()
    b.backward()
    b.check_backward()


@pytest.mark.parametrize("counts", [(1, 15, 16, 17, 31, 32, 33, 47, 63, 64, 65, 96, 97, 128, 129, 160, 161, 192, 193, 225),
                                    (257, 300, 0, 385, 511, 2, 640, 225, 513, 64, 255, 1, 100, 0, 31, 448, 7, 700, 321, 150)])
@pytest.mark.parametrize("d,f", [(4032, 192), (192, 4032)])
def test_chunks_of_every_length(counts, d, f):
    """So many columns that chunks are not made shorter to fill the chip."""
    idx = torch.cat([torch.full((n,), e) for e, n in enumerate(counts)])
    idx = idx[torch.randperm(len(idx), generator=torch.Generator().manual_seed(f))].reshape(-1, 1).cuda()
    b = Block(d + counts[0], len(idx), d, f, 20, 1, idx=idx)
    b.forward()
    b.check_forward()
    b.grads(torch.float16)
    b.backward()
    b.check_backward()


def test_rows_of_one_expert_past_32_bits():
    """Hidden rows of one expert that lie further apart than 2^32 bytes: gradients of the matrices, the last 64 hidden columns."""
    T, d, f, n = 140000, 64, 16384, 64
    idx = torch.zeros(T, 1, dtype=torch.int32, device="cuda")
    idx[-100:] = 1
    b = Block(85, T, d, f, 2, 1, idx=idx)
    b.forward()
    b.grads()
    b.backward()
    cols = slice(f - n, f)
    ref = Ref(b.x, b.w1[:, cols], b.w3[:, cols], b.w2[:, :, cols], list(b.perm.long().split(b.counts)), b.gate.double().reshape(-1), 1)
    r = ref.backward(b.a[:, cols], b.u[:, cols], b.d_out)
    for e in range(2):
        assert_within(b.g1[e, cols], *r["w1"][e], "w1")
        assert_within(b.g3[e, cols], *r["w3"][e], "w3")
        assert_within(b.g2[e, :, cols], *r["w2"][e], "w2")
