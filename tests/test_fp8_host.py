"""Products in 8-bit floating point and the training of the gate, host side: argument checks of the C-ABI and of the binding, workspace
arithmetic, and the reference's own rounding.  No kernel is launched here."""
import ctypes

import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm
from tests import fp8_ref


@pytest.fixture(scope="module")
def L():
    return mm.lib()


def _layer(prec=mm.PREC_FP16, d=256, f=512, E=4, k=2, resident=0, scale=4096, zero=None):
    ex = (mm.CExpert * E)()
    for e in ex:
        e.prec, e.resident = prec, resident
        for m in (e.w1, e.w3, e.w2):
            m.data, m.scale, m.zero = 4096, scale, zero
    return mm.CLayer(d, f, E, k, 4096, None, ex)


def test_reference_rounding_is_the_one_of_torch():
    v = np.concatenate([np.random.default_rng(0).standard_normal(4096) * s for s in (1e-3, 0.01, 1.0, 100.0)])
    v = np.clip(v.astype(np.float32), -448, 448)
    ties = (fp8_ref.VALUES[:0x7E] + fp8_ref.VALUES[1:0x7F]) / 2
    v = np.concatenate([v, ties, -ties, fp8_ref.VALUES[:0x7F]]).astype(np.float32)
    want = torch.from_numpy(v).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(fp8_ref.e4m3_codes(v.astype(np.float64)), want)
    got = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy()
    assert np.array_equal(got, fp8_ref.VALUES.astype(np.float32), equal_nan=True)


def test_experts_of_this_form_need_scales_and_no_zeros(L):
    ok, bad = _layer(mm.PREC_FP8B128, resident=1), _layer(mm.PREC_FP8B128, resident=1, scale=None)
    assert L.moe_route(ctypes.byref(ok), None, 1, 1, 1, None) == mm.MOE_EINVAL and b"NULL" in L.moe_last_error()
    assert L.moe_route(ctypes.byref(bad), 4096, 1, 1, 1, None) == mm.MOE_EINVAL and b"scale" in L.moe_last_error()
    ok.experts[1].prec = 4
    assert L.moe_route(ctypes.byref(ok), 4096, 1, 1, 1, None) == mm.MOE_EINVAL and b"precision" in L.moe_last_error()


def test_workspace_holds_quantized_rows(L):
    for T in (1, 7, 300):
        plain, fp8 = _layer(), _layer(mm.PREC_FP8B128)
        P = 2 * T
        rows = P * (256 + 512) + P * 4 * (2 + 4)
        got = L.moe_workspace_bytes(ctypes.byref(fp8), T)
        # no partial results of split contractions, room for codes and scales
        hidden = P * 512 * 2 + P * 256 * 4
        assert got >= rows + hidden and got % 256 == 0
        mixed = _layer()
        mixed.experts[3].prec = mm.PREC_FP8B128
        assert L.moe_workspace_bytes(ctypes.byref(mixed), T) == got
        assert L.moe_workspace_bytes(ctypes.byref(plain), T) > 0
        assert L.moe_layer_forward(ctypes.byref(fp8), 4096, T, 4096, None, None, 4096, got - 1, None) == mm.MOE_EWORKSPACE


def test_a_chain_needs_the_room_of_its_largest_layer(L):
    layers = (mm.CLayer * 2)(_layer(), _layer(mm.PREC_FP8B128))
    gains = (ctypes.c_void_p * 2)(4096, 4096)
    least = L.moe_workspace_bytes(ctypes.byref(layers[1]), 4)
    assert L.moe_chain_forward(layers, gains, 2, 1e-5, 4096, 4, None, 4096, least - 1, None) == mm.MOE_EWORKSPACE


def test_swap_slots_hold_the_form(L):
    slot = L.moe_swap_slot_bytes(ctypes.byref(_layer(mm.PREC_FP8B128, d=320, f=704)))
    assert slot >= 3 * 320 * 704 + 4 * (2 * 6 * 3 + 3 * 6) and slot % 256 == 0


def test_products_refuse(L):
    m = (mm.CMat * 2)(mm.CMat(4096, 4096, None), mm.CMat(4096, 4096, None))
    one = ctypes.byref(m[0])
    call = L.moe_matmul_fp8
    assert call(one, 16, 24, 4096, 4096, 1, 4096, 0, None) == mm.MOE_ESHAPE          # in: a multiple of 16
    assert call(one, -1, 32, 4096, 4096, 1, 4096, 0, None) == mm.MOE_EINVAL
    assert call(one, 16, 32, 4096, 4096, -1, 4096, 0, None) == mm.MOE_EINVAL
    assert call(one, 16, 32, 4096, 4096, (1 << 20) + 1, 4096, 0, None) == mm.MOE_ESHAPE
    assert call(one, 16, (1 << 20) + 16, 4096, 4096, 1, 4096, 0, None) == mm.MOE_ESHAPE
    assert call(one, 16, 32, 4096, 4096, 1, 4096, 2, None) == mm.MOE_EINVAL          # y_type
    assert call(one, 16, 32, 4096 + 8, 4096, 1, 4096, 0, None) == mm.MOE_EINVAL      # alignment
    assert call(one, 16, 32, None, 4096, 1, 4096, 0, None) == mm.MOE_EINVAL
    assert call(None, 16, 32, 4096, 4096, 1, 4096, 0, None) == mm.MOE_EINVAL
    assert call(one, 16, 32, None, None, 0, None, 0, None) == mm.MOE_OK              # nothing to do
    assert L.moe_quantize_fp8_rows(None, 0, 32, None, None, None) == mm.MOE_OK
    assert L.moe_quantize_fp8(None, 0, 32, None, None, None) == mm.MOE_OK
    assert call(ctypes.byref(mm.CMat(4096, None, None)), 16, 32, 4096, 4096, 1, 4096, 0, None) == mm.MOE_EINVAL
    assert call(ctypes.byref(mm.CMat(4104, 4096, None)), 16, 32, 4096, 4096, 1, 4096, 0, None) == mm.MOE_EINVAL
    group = L.moe_matmul_fp8_grouped
    for E, off, perm, k, rows, pairs, want in ((0, 4096, 4096, 1, 4, 4, mm.MOE_ESHAPE), (33, 4096, 4096, 1, 4, 4, mm.MOE_ESHAPE),
                                               (2, None, 4096, 1, 4, 4, mm.MOE_EINVAL), (2, 4096, 4096, 0, 4, 4, mm.MOE_ESHAPE),
                                               (2, 4096, None, 1, 3, 4, mm.MOE_ESHAPE), (2, 4096, 4096, 1, 0, 4, mm.MOE_ESHAPE)):
        assert group(m, E, 16, 32, 4096, 4096, rows, off, perm, k, pairs, 4096, 0, None) == want
    assert L.moe_quantize_fp8(4096, 16, 40, 4096, 4096, None) == mm.MOE_ESHAPE
    assert L.moe_quantize_fp8(4096, 16, 48, 4100, 4096, None) == mm.MOE_EINVAL
    assert L.moe_quantize_fp8_rows(4096, 2, 40, 4096, 4096, None) == mm.MOE_ESHAPE
    assert L.moe_quantize_fp8_rows(4096, -2, 48, 4096, 4096, None) == mm.MOE_EINVAL
    assert L.moe_quantize_fp8_rows(None, 2, 48, 4096, 4096, None) == mm.MOE_EINVAL
    assert L.moe_transpose_fp8(one, 24, 32, 4096, 4096, None) == mm.MOE_ESHAPE
    assert L.moe_dequant_fp8(one, 16, 32, 4096 + 2, None) == mm.MOE_EINVAL


def test_gate_calls_refuse(L):
    lay = _layer()
    p = ctypes.byref(lay)
    ws = L.moe_gate_workspace_bytes(p, 9)
    assert ws > 0 and L.moe_gate_workspace_bytes(p, 0) == 0 and L.moe_gate_workspace_bytes(None, 9) == 0
    assert L.moe_route_logits(p, 4096, 9, None, 4096, 4096, None) == mm.MOE_EINVAL
    assert L.moe_route_logits(p, 4096, 0, 4096, 4096, 4096, None) == mm.MOE_ESHAPE
    loss = L.moe_balance_loss
    assert loss(p, 4096, 4096, None, 9, 4096, 4096, 4096, None, 0, None) == mm.MOE_EWORKSPACE
    assert loss(p, 4096, 4096, None, 9, 4096, 4096, 4096, 4096, ws - 1, None) == mm.MOE_EWORKSPACE
    assert loss(p, 4096, 4096, None, 9, 4096, 4096, 4096, 4096 + 16, ws, None) == mm.MOE_EWORKSPACE
    assert loss(p, 4096, 4096, None, 0, 4096, 4096, 4096, 4096, ws, None) == mm.MOE_ESHAPE
    assert loss(p, None, 4096, None, 9, 4096, 4096, 4096, 4096, ws, None) == mm.MOE_EINVAL

    def back(x=4096, logits=4096, T=9, counts=4096, d_gate=4096, d_loss=4096, dl=4096, dx=4096, kind=0, dw=4096, db=4096, ws_bytes=ws):
        return L.moe_route_backward(p, x, logits, 4096, None, T, counts, d_gate, d_loss, dl, dx, kind, dw, db, 4096, ws_bytes, None)
    assert back(d_gate=None, d_loss=None, counts=None) == mm.MOE_EINVAL
    assert back(counts=None) == mm.MOE_EINVAL and back(d_loss=None) == mm.MOE_EINVAL
    assert back(dl=None, dx=None, dw=None, db=None) == mm.MOE_EINVAL
    assert back(x=None) == mm.MOE_EINVAL and back(kind=2) == mm.MOE_EINVAL and back(logits=None) == mm.MOE_EINVAL
    assert back(T=0) == mm.MOE_ESHAPE and back(ws_bytes=ws - 1) == mm.MOE_EWORKSPACE


def test_binding_refuses_before_the_library():
    """Types, shapes, strides and places of tensors (all of these are on the CPU, so a tensor that fits is refused for its place)."""
    codes, scale = torch.zeros(32, 48, dtype=torch.uint8), torch.zeros(1, 1)
    x8, xs, y = torch.zeros(3, 48, dtype=torch.uint8), torch.zeros(1, 3), torch.zeros(3, 32)

    def refused(code, f, *a, **k):
        with pytest.raises(mm.MoeError) as e:
            f(*a, **k)
        assert e.value.code == code, e.value
    refused(mm.MOE_EINVAL, mm.moe_matmul_fp8, mm.Mat(codes, scale), x8, xs, y)                       # not on a GPU
    refused(mm.MOE_EINVAL, mm.moe_matmul_fp8, mm.Mat(codes.float(), scale), x8, xs, y)
    refused(mm.MOE_EINVAL, mm.moe_quantize_fp8_rows, torch.zeros(3, 48), x8, xs)                     # fp32 rows
    refused(mm.MOE_EINVAL, mm.moe_quantize_fp8_rows, torch.zeros(48, 3, dtype=torch.float16).t(), x8, xs)
    refused(mm.MOE_ESHAPE, mm.moe_quantize_fp8_rows, torch.zeros(48, dtype=torch.float16), x8, xs)
    refused(mm.MOE_ESHAPE, mm.MatGroup, [])
    refused(mm.MOE_EINVAL, mm.MatGroup, [mm.Mat(codes, scale.double())])
    if not torch.cuda.is_available():
        refused(mm.MOE_EINVAL, mm.moe_dequant_fp8, mm.Mat(codes, scale), 32, 48, torch.zeros(32, 48, dtype=torch.float16))
