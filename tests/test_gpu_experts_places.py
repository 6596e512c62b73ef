"""Training of the experts: results that take the place of inputs which are needed no more have the bits that they have anywhere else."""
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm
from tests.test_gpu_experts_train import Block

pytestmark = pytest.mark.gpu


def block(dtype=torch.float16):
    b = Block(101, 200, 64, 192, 3, 2)
    b.forward()
    b.grads(dtype)
    b.backward()
    return b, b.results()


@pytest.mark.parametrize("place", ["x", "d_out", "a", "u"])
def test_gradient_of_the_tokens(place):
    b, (d_x, d_gate, g1, g3, g2) = block()
    b.grads(torch.float16)
    to = getattr(b, place)
    b.d_x = to if to.shape == d_x.shape else to.reshape(-1)[: d_x.numel()].reshape(d_x.shape)
    b.backward()
    assert all(torch.equal(p, q) for p, q in zip(b.results(), (d_x, d_gate, g1, g3, g2)))


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
def test_gradients_of_the_matrices_in_the_place_of_the_kept_rows(dtype):
    b, want = block(dtype)
    b.grads(dtype)
    n = b.d * b.f
    rows = [[b.g1[e], b.g3[e], b.g2[e]] for e in range(3)]
    for e, m, kept, i in ((0, 0, b.a, 0), (0, 2, b.a, 1), (1, 1, b.u, 0), (2, 2, b.u, 1)):
        rows[e][m] = kept.reshape(-1).view(dtype)[i * n: (i + 1) * n].reshape(rows[e][m].shape)
    b.d_w = mm.ExpertGrads(rows)
    b.backward()
    for e in range(3):
        for m in range(3):
            assert torch.equal(rows[e][m], want[2 + m][e])
    assert torch.equal(b.d_x, want[0]) and torch.equal(b.d_gate, want[1])


def test_gradients_of_the_gates_in_the_place_of_the_gates():
    b, want = block()
    b.grads(torch.float16)
    b.d_gate = b.gate
    b.backward()
    assert all(torch.equal(p, q) for p, q in zip(b.results(), want))
