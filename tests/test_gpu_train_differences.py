"""Gradients of the experts against differences of the output in 64 bits, along directions in which a wrong one shows (test_train_differences_host.py)."""
import pytest

torch = pytest.importorskip("torch")

from tests.test_gpu_experts_train import Block, gen
from tests.train_differences import LIMIT, WHAT, worst

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,d,f,E,k", [(50, 64, 128, 3, 2), (150, 192, 64, 2, 1), (9, 128, 320, 5, 4)])
@pytest.mark.parametrize("gone", [0.0, 0.3])
def test_gradients_against_differences(T, d, f, E, k, gone):
    idx = torch.rand(T, E, generator=gen(T), device="cuda").topk(k, 1).indices
    idx[torch.rand(T, generator=gen(d), device="cuda") < gone] = -1
    b = Block(41 + T, T, d, f, E, k, idx=idx)
    b.forward()
    b.grads()
    b.backward()
    formula = b.ref().backward(b.a, b.u, b.d_out)
    for what, grad in zip(WHAT, (b.d_x, b.d_gate.reshape(-1), b.g1, b.g3, b.g2)):
        f64 = formula["d_x"][0] if what == "x" else formula["d_gate"][0] if what == "gate" else torch.stack([v for v, _ in formula[what]])
        off = worst(b.ref(), b.d_out, what, grad, f64)
        assert off <= LIMIT, f"{what}: {off:.3g}"
