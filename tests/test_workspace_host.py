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
