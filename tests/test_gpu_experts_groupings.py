"""Groupings that no moe_permute gives: what lies in a group and names a pair is computed, and nothing outside the arrays is touched, those of the workspace among them."""
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm
from tests.test_gpu_experts_train import Block
from tests.train_ref import Ref, assert_within

pytestmark = pytest.mark.gpu

T, D, F, E, K = 60, 64, 128, 4, 2
P, GUARD = T * K, 4096                                         # bytes on both sides of a tensor


class Guarded:
    """A tensor of `fill` between bytes that have to stay."""

    def __init__(self, shape, dtype, fill):
        n = torch.empty(0, dtype=dtype).element_size() * int(torch.tensor(shape).prod())
        self.bytes = torch.full((GUARD + n + GUARD,), 0x5A, dtype=torch.uint8, device="cuda")
        self.t = self.bytes[GUARD: GUARD + n].view(dtype).view(shape)
        self.t.fill_(fill)
        self.n = n

    def check(self, what):
        assert (self.bytes[:GUARD] == 0x5A).all() and (self.bytes[GUARD + self.n:] == 0x5A).all(), what


def guarded_block(seed, dtype):
    """A block whose results and workspace are Guarded, all filled with 7."""
    b = Block(seed, T, D, F, E, K)
    g = dict(a=Guarded((P, F), torch.float16, 7), u=Guarded((P, F), torch.float16, 7), out=Guarded((T, D), torch.float16, 7), d_x=Guarded((T, D), dtype, 7),
             d_gate=Guarded((T, K), torch.float32, 7), g1=Guarded((E, F, D), dtype, 7), g3=Guarded((E, F, D), dtype, 7), g2=Guarded((E, D, F), dtype, 7),
             ws=Guarded((mm.experts_workspace_bytes(b.layer, T),), torch.uint8, 7))
    for name, v in g.items():
        setattr(b, name, v.t)
    b.d_w = mm.ExpertGrads([(b.g1[e], b.g3[e], b.g2[e]) for e in range(E)])
    return b, g


def run(b, g, offsets, perm):
    b.forward(offsets=offsets, perm=perm)
    b.backward(offsets=offsets, perm=perm)
    torch.cuda.synchronize()
    for name, v in g.items():
        v.check(name)


def check(b, offsets, perm):
    """Against the groups that are left: offsets within [0, P] and increasing, rows that name a pair."""
    at = [max(0, min(P, v)) for v in offsets]
    for i in range(E):
        at[i + 1] = max(at[i], at[i + 1])
    perm = torch.arange(P, device="cuda") if perm is None else perm.long()
    is_pair = (perm >= 0) & (perm < P)
    rows = [[r for r in range(at[e], at[e + 1]) if is_pair[r]] for e in range(E)]
    every = sum(rows, [])
    assert (b.a[: at[0]] == 7).all() and (b.a[at[E]:] == 7).all() and (b.u[: at[0]] == 7).all() and (b.u[at[E]:] == 7).all()
    ref = Ref(b.x, b.w1, b.w3, b.w2, [perm[r].long() for r in rows], b.gate.double().reshape(-1), K)
    (a, ea), (u, eu), (out, eo) = ref.forward()
    if every:
        assert_within(b.a[every], a, ea, "a")
        assert_within(b.u[every], u, eu, "u")
    assert_within(b.out, out, eo, "out")
    half = b.d_x.dtype == torch.float16
    r = ref.backward(b.a[every], b.u[every], b.d_out)
    assert_within(b.d_gate, *[v.reshape(T, K) for v in r["d_gate"]], "d_gate")
    assert_within(b.d_x, *r["d_x"], "d_x", half)
    for name, got in (("w1", b.g1), ("w3", b.g3), ("w2", b.g2)):
        for e in range(E):
            assert_within(got[e], *r[name][e], f"{name} of expert {e}", half)
            if not rows[e]:
                assert (got[e] == 0).all()
    without = torch.ones(P, dtype=torch.bool, device="cuda")
    without[perm[every]] = False
    assert (b.d_gate.reshape(-1)[without] == 0).all()
    none = without.reshape(T, K).all(1)
    assert (b.out[none] == 0).all() and (b.d_x[none] == 0).all()


OFFSETS = [[-7, 200, 50, 1000, 2 ** 31 - 1], [0, 90, 30, 20, 10], [5, 5, 5, 5, 5], [10, 20, 60, 61, 100], [-2 ** 31, -5, -1, 0, 0], [P, P, P, P, P], [33, 2, 97, 2 ** 31 - 1, -2 ** 31],
           [0, 0, 0, 0, P], [119, 120, 120, 120, 121]]


@pytest.mark.parametrize("offsets", OFFSETS, ids=str)
@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_offsets_that_are_none(offsets, dtype):
    b, g = guarded_block(8, dtype)
    run(b, g, torch.tensor(offsets, dtype=torch.int32, device="cuda"), b.perm)
    check(b, offsets, b.perm)


def test_offsets_that_are_none_without_perm():
    for offsets in OFFSETS:
        b, g = guarded_block(9, torch.float32)
        run(b, g, torch.tensor(offsets, dtype=torch.int32, device="cuda"), None)
        check(b, offsets, None)


@pytest.mark.parametrize("bad", [-1, -2 ** 31, P, 2 ** 31 - 1])
def test_rows_that_name_no_pair(bad):
    """Every third row: what is left is computed as if these were not there."""
    b, g = guarded_block(10, torch.float32)
    perm = b.perm.clone()
    perm[::3] = bad
    run(b, g, b.offsets, perm)
    check(b, b.offsets.tolist(), perm)


def test_no_row_names_a_pair():
    b, g = guarded_block(11, torch.float32)
    perm = torch.randint(P, 2 ** 31 - 1, (P,), device="cuda", dtype=torch.int32)
    run(b, g, b.offsets, perm)
    for t in (b.out, b.d_x, b.d_gate, b.g1, b.g3, b.g2):
        assert (t == 0).all()


def test_a_pair_in_every_row():
    """Pair 0 in the groups of all experts: its token gets one of its rows, nobody else gets anything."""
    b, g = guarded_block(12, torch.float32)
    perm = torch.zeros(P, dtype=torch.int32, device="cuda")
    run(b, g, b.offsets, perm)
    assert (b.out[1:] == 0).all() and (b.d_x[1:] == 0).all() and (b.d_gate.reshape(-1)[1:] == 0).all()
    outs = [Ref(b.x, b.w1, b.w3, b.w2, [torch.tensor([0] if i == e else [], dtype=torch.long, device="cuda") for i in range(E)], b.gate.double().reshape(-1), K).forward()[2]
            for e in range(E)]
    assert any(((b.out[0].double() - v[0]).abs() <= bound[0]).all() for v, bound in outs)
