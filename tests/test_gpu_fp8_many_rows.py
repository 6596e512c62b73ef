"""e4m3 experts and products with as many rows as the tile kernel takes: results against 64 bits, and what a call leaves in its workspace against the
quantizers."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm
from tests import fp8_ref
from tests.common import unsplit_workspace_bytes
from tests.gpu_common import dev
from tests.test_gpu_fp8 import check_product, normal, on_device, quantized_matrix, rng_of, rows_per_chunk, spoiled

pytestmark = pytest.mark.gpu


def quantized_of(ws, d, f, E, k, T, rows, x_rows):
    """Codes and scales that the last call on T tokens left of its tokens (x_rows) and its hidden rows: they lie behind what every workspace holds."""
    raw, at, got = ws.cpu().numpy(), unsplit_workspace_bytes(d, f, E, k, T), []
    for width, n in ((d, x_rows), (f, rows)):
        b, P = -(-width // 128), T * k
        codes = raw[at:at + n * width].reshape(n, width)
        at += -(-P * width // 256) * 256
        got.append((codes, raw[at:at + 4 * b * n].view(np.float32).reshape(b, n)))
        at += -(-P * 4 * b // 256) * 256
    return got


def expert_of(rng, d, f, scale=0.05):
    mats = [quantized_matrix(rng, o, i, scale) for o, i in ((f, d), (f, d), (d, f))]
    return mm.Expert(mm.PREC_FP8B128, *[on_device(m) for m in mats]), mats


@pytest.mark.parametrize("n,d,f", [(600, 2112, 3008), (1000, 1408, 2816), (300, 1408, 4096)])
def test_rows_of_an_expert_alone_are_sums_in_32_bits(n, d, f):
    """fp32 rows are the products of the quantized hidden rows as exact as 32 bits allow, for many rows as for few."""
    assert rows_per_chunk(n, d, f, exact=True) and rows_per_chunk(n, d, f)
    print(f"expert alone {n} rows {d} x {f}", flush=True)
    rng = rng_of(n, d, f, 31)
    ex, mats = expert_of(rng, d, f)
    gone = mm.Expert(mm.PREC_FP16, None, None, None, resident=False)
    layer = mm.Layer(d, f, 2, dev(normal(rng, 2, d)), [gone, ex])
    T = -(-n // 2)
    x, ws, y = normal(rng, n, d), mm.alloc_workspace(layer, T), spoiled((n, d), torch.float32)
    mm.moe_expert_ffn_mixed(layer, 1, dev(x), y, ws)
    (x8, xs), (h8, hs) = quantized_of(ws, d, f, 2, 2, T, n, n)
    want, want_scale = fp8_ref.quantize_rows(x)
    assert np.array_equal(x8, want) and np.array_equal(xs, want_scale)
    check_product(y.cpu().numpy(), fp8_ref.row_values(h8, hs), fp8_ref.matrix_values(*mats[2]), f, False, (n, d, f))
