"""Sizes of workspaces and of calls, host side: tables of experts that are not there yet, sizes past what one launch can do.  No kernel is launched here."""
import ctypes

import pytest

from paper_2407_14417_amd import binding as mm
from tests.common import unsplit_workspace_bytes


@pytest.fixture(scope="module")
def L():
    return mm.lib()


def layer_of(precs, d, f, k, n_experts=None):
    if precs is None:
        return mm.CLayer(d, f, n_experts, k, 4096, None, None)
    ex = (mm.CExpert * len(precs))()
    for e, p in zip(ex, precs):
        e.prec = p
    return mm.CLayer(d, f, len(precs), k, 4096, None, ex)


@pytest.mark.parametrize("d,f,E,k", [(256, 512, 4, 2), (4096, 14336, 8, 2), (1088, 3008, 8, 2), (64, 64, 1, 1), (320, 2304, 32, 8), (512, 2880, 4, 2)])
def test_a_workspace_for_a_table_that_is_not_there_yet(L, d, f, E, k):
    """It serves every table of the shape; the bytes for a table that is there are those of its precisions."""
    for T in (1, 2, 7, 16, 40, 96, 130, 512, 2000):
        size = lambda precs: L.moe_workspace_bytes(ctypes.byref(layer_of(precs, d, f, k, E)), T)  # noqa: E731
        filled = [size([p] * E) for p in (mm.PREC_FP16, mm.PREC_INT4G64, mm.PREC_INT8G64, mm.PREC_FP8B128)]
        mixed = size([mm.PREC_FP8B128] + [mm.PREC_INT4G64] * (E - 1))
        assert filled[0] == filled[1] == filled[2] and mixed == filled[3]
        assert filled[0] >= unsplit_workspace_bytes(d, f, E, k, T) and filled[3] > unsplit_workspace_bytes(d, f, E, k, T)
        for unknown in (None, [0x5A5A5A5A] * E, [mm.PREC_FP8B128] * (E - 1) + [-1], [mm.PREC_FP16] * (E - 1) + [4]):
            assert size(unknown) == max(filled), (T, unknown)


def test_binding_asks_for_any_precision():
    gone = [mm.Expert(mm.PREC_FP16, None, None, None, resident=False) for _ in range(4)]
    layer = mm.Layer(256, 512, 2, None, gone)
    later = mm.Layer(256, 512, 2, None, gone[:3] + [mm.Expert(mm.PREC_FP8B128, None, None, None, resident=False)])
    for T in (1, 40):
        plain, most = mm.workspace_bytes(layer, T), mm.workspace_bytes(layer, T, any_precision=True)
        assert most == max(plain, mm.workspace_bytes(later, T)) == mm.workspace_bytes(later, T, any_precision=True)


def test_sizes_past_one_launch_are_refused(L):
    """A launch has less than 2^32 threads along its first dimension and 2^16 workgroups along its second: larger calls are refused before it."""
    most = 2 ** 29 - 32                                      # blocks of 128 columns of all rows, eight threads each
    n = most // 8192 + 1
    assert L.moe_quantize_fp8_rows(4096, n, 1 << 20, 4096, 4096, None) == mm.MOE_ESHAPE and b"moe_quantize_fp8_rows" in L.moe_last_error()
    assert L.moe_quantize_fp8_rows(4096, 1 << 22, 128 * 128, 4096, 4096, None) == mm.MOE_ESHAPE
    m = ctypes.byref(mm.CMat(4096, 4096, None))
    assert L.moe_dequant_fp8(m, 1 << 18, 1 << 17, 4096, None) == mm.MOE_ESHAPE and b"moe_dequant_fp8" in L.moe_last_error()
    assert L.moe_dequant_fp8(m, 1 << 20, 1 << 20, 4096, None) == mm.MOE_ESHAPE
    lay = layer_of([mm.PREC_FP8B128] * 8, 64, 64, 8)
    p, T = ctypes.byref(lay), (63 << 16) // 8 + 1            # (token, slot) pairs of a block with e4m3 experts
    assert L.moe_layer_forward(p, 4096, T, 4096, None, None, 4096, 1 << 62, None) == mm.MOE_ESHAPE
    assert L.moe_layer_forward(p, 4096, T - 1, 4096, None, None, 4096, 4096, None) == mm.MOE_EWORKSPACE
    assert L.moe_route_logits(p, 4096, 1 << 24, 4096, 4096, 4096, None) == mm.MOE_ESHAPE
    ws = 1 << 62
    assert L.moe_balance_loss(p, 4096, 4096, None, 1 << 28, 4096, 4096, 4096, 4096, ws, None) == mm.MOE_ESHAPE    # 2^31 pairs
    # tokens up to the last int: as many shares of d_w, one float per expert and token more (64 tokens are 2048 bytes)
    assert 0 < L.moe_gate_workspace_bytes(p, 2 ** 31 - 1) < ws
    assert L.moe_gate_workspace_bytes(p, 2 ** 31 - 1) - L.moe_gate_workspace_bytes(p, 2 ** 31 - 64) == 64 * 8 * 4


def test_d_x_on_x_is_refused(L):
    """Tokens are read for d_w_gate while rows of d_x are written: not in place, nor with a part of the rows."""
    lay = layer_of([mm.PREC_FP16] * 4, 64, 64, 2)
    p, T, d, x = ctypes.byref(lay), 9, 64, 1 << 20

    ws = L.moe_gate_workspace_bytes(p, T)
    for kind, size in ((mm.OUT_F16, 2), (mm.OUT_F32, 4)):
        for dx in (x, x + T * d * 2 - 2, x - T * d * size + 2):
            rc = L.moe_route_backward(p, x, 4096, 4096, None, T, None, 4096, None, None, dx, kind, 4096, None, 4096, ws, None)
            assert rc == mm.MOE_EINVAL and b"d_x" in L.moe_last_error()
