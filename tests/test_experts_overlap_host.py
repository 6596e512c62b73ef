"""Training of the experts, clipping: results in places that a call reads until its end are refused.  No call here reaches a launch."""
import ctypes

import pytest

from paper_2407_14417_amd import binding as mm
from tests.test_built_code import LIB

pytestmark = pytest.mark.skipif(not LIB.exists(), reason="needs the built library")

D, F, E, K, T = 128, 192, 3, 2, 10
PLACE = 1 << 24                                                # between tensors that do not overlap
NAMES = ("x", "gate", "offsets", "perm", "a", "u", "out", "d_out", "d_x", "d_gate", "ws") + tuple(f"{m}{e}" for e in range(E) for m in ("w1", "w3", "w2"))
AT = {name: (i + 1) * PLACE for i, name in enumerate(NAMES)}
MATRIX, ROWS, KEPT = D * F * 2, T * D * 2, T * K * F * 2
# what lies there, in bytes
SIZE = dict(x=ROWS, gate=T * K * 4, offsets=(E + 1) * 4, perm=T * K * 4, a=KEPT, u=KEPT, out=ROWS, d_out=ROWS, d_x=T * D * 4, d_gate=T * K * 4) | {
    n: MATRIX for n in NAMES if n[0] == "w" and n != "ws"}


def layer():
    mats = [[mm.CMat(AT[f"{m}{e}"], None, None) for m in ("w1", "w3", "w2")] for e in range(E)]
    return mm.CLayer(D, F, E, K, None, None, (mm.CExpert * E)(*[mm.CExpert(mm.PREC_FP16, 1, *m) for m in mats]))


def places(name, size, align=16):
    """Addresses at which `size` bytes and the tensor of that name have their first or last bytes in common."""
    first = -(-(AT[name] - size + 1) // align) * align
    last = (AT[name] + SIZE.get(name, mm.lib().moe_experts_workspace_bytes(layer(), T)) - 1) // align * align
    return first, AT[name], last


def backward(grads=(), kind=0, **at):
    """grads: (expert, matrix, address)"""
    table = [[None] * 3 for _ in range(E)]
    for e, m, p in grads:
        table[e][m] = p
    d_w = (mm.CExpertGrads * E)(*[mm.CExpertGrads(*g) for g in table])
    p = AT | at
    L = layer()
    return mm.lib().moe_experts_backward(ctypes.byref(L), p["x"], T, p["gate"], p["offsets"], p["perm"], p["a"], p["u"], p["d_out"], p["d_x"], 0, p["d_gate"],
                                         d_w if grads else None, kind, 0, p["ws"], 1 << 40, None)


def forward(**at):
    p = AT | at
    L = layer()
    return mm.lib().moe_experts_forward(ctypes.byref(L), p["x"], T, p["gate"], p["offsets"], p["perm"], p["a"], p["u"], p["out"], p["ws"], 1 << 40, None)


def refused(rc):
    return rc == mm.MOE_EINVAL and b"overlap" in mm.lib().moe_last_error()


@pytest.mark.parametrize("kind", [0, 1])
@pytest.mark.parametrize("m", [0, 1, 2])
@pytest.mark.parametrize("over", ["x", "d_out", "offsets", "perm", "ws", "d_x", "d_gate", "w10", "w32", "w21"])
def test_gradients_of_matrices_over_what_is_still_read(over, m, kind):
    """They are written beside reads of x, d_out and the grouping, and before the matrices and the workspace are read for d_x."""
    for p in places(over, MATRIX * (1 if kind else 2)):
        assert refused(backward([(1, m, p)], kind))


@pytest.mark.parametrize("name", ["d_x", "d_gate"])
@pytest.mark.parametrize("over", ["offsets", "perm", "ws", "w10", "w32", "w21"])
def test_gradients_of_tokens_and_gates_over_what_is_still_read(over, name):
    align = 16 if name == "d_x" else 4
    for p in places(over, SIZE[name], align):
        assert refused(backward(**{name: p}))
    for p in places("d_x", SIZE["d_gate"], 4):
        assert refused(backward(d_gate=p))


@pytest.mark.parametrize("name", ["a", "u", "out"])
@pytest.mark.parametrize("over", ["x", "offsets", "perm", "ws", "w10", "w32", "w21", "a", "u", "out"])
def test_results_of_the_forward_pass_over_what_is_still_read(over, name):
    """(out may lie over x)"""
    if name != over and (name, over) != ("out", "x"):
        for p in places(over, SIZE[name]):
            assert refused(forward(**{name: p}))


def clip(entries, norm=AT["d_gate"], ws=AT["ws"]):
    return mm.lib().moe_clip_gradients((mm.CGrad * len(entries))(*[mm.CGrad(*e) for e in entries]), len(entries), 1.0, 1.0, norm, ws, 1 << 40, None)


@pytest.mark.parametrize("n", [1, 100, 200000])                # one workgroup, two launches
@pytest.mark.parametrize("kind", [0, 1])
def test_norm_and_workspace_of_clipping_over_a_tensor(n, kind):
    """The norm is written while gradients are read and outs written; the workspace holds sums in between."""
    g, o, size = AT["x"], AT["out"], n * (2 if kind else 4)
    room = mm.lib().moe_clip_workspace_bytes(2)
    other = (AT["a"], AT["u"], 10, 0, 0)
    for entries in ([(g, o, n, kind, kind), other], [other, (g, g, n, kind, kind)]):
        for tensor in {entries[0][0], entries[0][1], entries[1][0], entries[1][1]} & {g, o}:
            last = tensor + size - 1
            for norm in (tensor, last // 4 * 4):
                assert refused(clip(entries, norm=norm))
            for ws in (tensor, last // 256 * 256, (tensor - room) // 256 * 256 + 256):
                assert refused(clip(entries, ws=ws))
    assert refused(clip([other], norm=AT["ws"] + 8))


def test_a_gradient_that_is_none():
    """A parameter without one is the caller's to leave out; the error is the binding's."""
    torch = pytest.importorskip("torch")
    for grads, outs in (([None], None), ([None], [torch.zeros(3)])):
        with pytest.raises(mm.MoeError) as e:
            mm.GradList(grads, outs)
        assert e.value.code == mm.MOE_EINVAL and "gradient 0" in str(e.value)
