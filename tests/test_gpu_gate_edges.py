"""The gate's backward pass where inputs are not finite or outputs overlap inputs."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm
from tests.test_gpu_gate_grad import ALL, case, cuda, gate_layer, loss_of, run_backward

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,E,k,d", [(37, 6, 2, 192), (700, 32, 4, 256)])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("want", [ALL, ("d_x",)])
def test_rows_of_padding_get_zeros_whatever_the_gate_holds(T, E, k, d, half, want):
    rng = np.random.default_rng([T, E, k, d])
    z, idx, valid = case(rng, T, E, k, 0.4)
    x, w = rng.standard_normal((T, d)).astype(np.float16), (rng.standard_normal((E, d)) * 0.05).astype(np.float16)
    dg = rng.standard_normal((T, k)).astype(np.float32)
    counts, _, _ = loss_of(z.astype(np.float64), idx, valid, E, k)
    kind, xs = torch.float16 if half else torch.float32, x if "d_w_gate" in want else None
    clean = run_backward(gate_layer(E, k, d, cuda(w)), xs, z, idx, valid, counts, dg, 7.0, want, kind)
    bad = w.copy()
    bad[2, 5], bad[0, 77], bad[E - 1, d - 1] = np.inf, np.nan, -np.inf
    got = run_backward(gate_layer(E, k, d, cuda(bad)), xs, z, idx, valid, counts, dg, 7.0, want, kind)
    assert np.all(got["d_x"][valid == 0] == 0) and np.all(clean["d_x"][valid == 0] == 0)
    live, cols = valid == 1, [5, 77, d - 1]
    assert not np.isfinite(got["d_x"][live][:, cols]).any()
    assert np.array_equal(np.delete(got["d_x"], cols, 1), np.delete(clean["d_x"], cols, 1))
    for n in set(want) - {"d_x"}:
        assert np.array_equal(got[n], clean[n]), n
