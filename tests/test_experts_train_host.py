"""Training of the experts, norm and clipping: refusals and sizes, on the host.  No call here reaches a launch."""
import ctypes
import re
import subprocess

import pytest

from paper_2407_14417_amd import binding as mm
from tests.test_built_code import LIB, OBJDUMP, _code_objects

pytestmark = pytest.mark.skipif(not LIB.exists(), reason="needs the built library")

D, F, E, K, T = 128, 192, 3, 2, 10
AT = 1 << 20            # an aligned address that nothing reads


def layer(d=D, f=F, n=E, k=K, prec=mm.PREC_FP16, resident=1, data=AT, table=True):
    m = mm.CMat(data, None, None)
    experts = (mm.CExpert * max(n, 1))(*[mm.CExpert(prec, resident, m, m, m) for _ in range(max(n, 1))])
    return mm.CLayer(d, f, n, k, None, None, experts if table else None)


def forward(L, T=T, x=AT, gate=AT, offsets=AT, perm=AT, a=2 * AT, u=3 * AT, out=4 * AT, ws=5 * AT, ws_bytes=1 << 40):
    return mm.lib().moe_experts_forward(L, x, T, gate, offsets, perm, a, u, out, ws, ws_bytes, None)


def backward(L, T=T, x=AT, gate=AT, offsets=AT, perm=AT, a=2 * AT, u=3 * AT, d_out=4 * AT, d_x=6 * AT, d_x_type=0, d_gate=AT, d_w=None, d_w_type=0, ws=5 * AT,
             ws_bytes=1 << 40):
    return mm.lib().moe_experts_backward(L, x, T, gate, offsets, perm, a, u, d_out, d_x, d_x_type, d_gate, d_w, d_w_type, 0, ws, ws_bytes, None)


@pytest.mark.parametrize("call", [forward, backward])
def test_refusals_of_both(call):
    for L, T_, want in ((None, T, mm.MOE_EINVAL), (layer(table=False), T, mm.MOE_EINVAL), (layer(d=96), T, mm.MOE_ESHAPE), (layer(f=0), T, mm.MOE_ESHAPE),
                        (layer(d=8256), T, mm.MOE_ESHAPE), (layer(f=16448), T, mm.MOE_ESHAPE), (layer(n=33, k=2), T, mm.MOE_ESHAPE), (layer(n=0), T, mm.MOE_ESHAPE),
                        (layer(k=4), T, mm.MOE_ESHAPE), (layer(k=0), T, mm.MOE_ESHAPE), (layer(), 0, mm.MOE_ESHAPE), (layer(), -3, mm.MOE_ESHAPE),
                        (layer(), (1 << 21) + 1, mm.MOE_ESHAPE), (layer(d=8192, k=1), 1 << 18, mm.MOE_ESHAPE), (layer(prec=mm.PREC_INT4G64), T, mm.MOE_EINVAL),
                        (layer(prec=mm.PREC_FP8B128), T, mm.MOE_EINVAL), (layer(resident=0), T, mm.MOE_ENOTRESIDENT), (layer(data=None), T, mm.MOE_ENOTRESIDENT),
                        (layer(data=AT + 8), T, mm.MOE_EINVAL)):
        assert call(None if L is None else ctypes.byref(L), T=T_) == want
        assert mm.lib().moe_last_error()
    L = layer()
    assert call(L, offsets=None) == mm.MOE_EINVAL
    for name in ("gate", "offsets", "perm"):
        assert call(L, **{name: AT + 2}) == mm.MOE_EINVAL
    for name in ("x", "a", "u"):
        assert call(L, **{name: None}) == mm.MOE_EINVAL and call(L, **{name: AT + 8}) == mm.MOE_EINVAL
    assert call(L, ws=None) == call(L, ws=AT + 128) == call(L, ws_bytes=T * K * (6 * F + 4 * D)) == mm.MOE_EWORKSPACE


def test_refusals_of_the_forward_pass():
    L = layer()
    assert forward(L, out=None) == forward(L, out=AT + 2) == mm.MOE_EINVAL
    kept, rows = T * K * F * 2, T * D * 2
    assert forward(L, a=2 * AT, u=2 * AT + kept - 16) == mm.MOE_EINVAL
    assert forward(L, a=AT + rows - 16) == forward(L, u=AT) == forward(L, out=2 * AT) == forward(L, out=3 * AT + kept - 16) == mm.MOE_EINVAL


def test_refusals_of_the_backward_pass():
    L = layer()
    assert backward(L, d_out=None) == backward(L, d_out=AT + 8) == mm.MOE_EINVAL
    assert backward(L, d_x=None, d_gate=None) == mm.MOE_EINVAL
    assert backward(L, d_x_type=2) == backward(L, d_w_type=-1) == mm.MOE_EINVAL
    assert backward(L, d_x=AT + 4) == backward(L, d_gate=AT + 2) == mm.MOE_EINVAL
    for i in range(3):
        entry = [AT, None, AT]
        entry[i] = AT + 8
        grads = (mm.CExpertGrads * E)(*[mm.CExpertGrads(None, None, None)] * 2, mm.CExpertGrads(*entry))
        assert backward(L, d_w=grads) == mm.MOE_EINVAL


def test_gradients_over_one_another():
    L, size = layer(), D * F * 4

    def says(*at, kind=0):
        entries = list(at) + [None] * (3 * E - len(at))
        return backward(L, d_w=(mm.CExpertGrads * E)(*[mm.CExpertGrads(*entries[3 * e: 3 * e + 3]) for e in range(E)]), d_w_type=kind)
    A = 16 * AT
    assert says(A, A) == says(A, None, A) == says(A, None, None, None, A) == mm.MOE_EINVAL                  # the same twice
    assert says(A, A + size - 16) == says(A + size - 16, None, None, A) == says(A, A + size // 2 - 16, kind=1) == mm.MOE_EINVAL
    assert says(4 * A, A, 2 * A, 3 * A, None, 4 * A + 16) == mm.MOE_EINVAL and b"overlap" in mm.lib().moe_last_error()


def test_workspace_bytes():
    ask = mm.lib().moe_experts_workspace_bytes
    assert ask(None, T) == ask(layer(), 0) == ask(layer(d=100), T) == 0
    # three sets of rows of d_ff in fp16 and one of d_model in fp32, at least
    for t in (1, 10, 1000, 100000):
        assert ask(layer(table=False), t) >= t * K * (6 * F + 4 * D)
    L = layer(d=8192, f=16384, n=32, k=8)
    assert ask(L, 1 << 17) >= (1 << 20) * (6 * 16384 + 4 * 8192)
    assert mm.lib().moe_clip_workspace_bytes(-1) == 0 and mm.lib().moe_clip_workspace_bytes(1025) == 0
    assert 0 < mm.lib().moe_clip_workspace_bytes(0) <= mm.lib().moe_clip_workspace_bytes(1024)


def clip(entries, n=None, max_norm=1.0, unscale=1.0, norm=AT, ws=5 * AT, ws_bytes=1 << 30):
    grads = (mm.CGrad * max(1, len(entries)))(*[mm.CGrad(*e) for e in entries])
    return mm.lib().moe_clip_gradients(grads, len(entries) if n is None else n, max_norm, unscale, norm, ws, ws_bytes, None)


def test_refusals_of_clipping():
    ok = (2 * AT, 3 * AT, 100, 0, 0)
    assert clip([ok], n=-1) == mm.MOE_EINVAL and clip([ok], n=1025) == mm.MOE_ESHAPE
    assert mm.lib().moe_clip_gradients(None, 1, 1.0, 1.0, AT, 5 * AT, 1 << 30, None) == mm.MOE_EINVAL
    assert clip([ok], norm=None) == clip([ok], norm=AT + 2) == mm.MOE_EINVAL
    for bad in (float("nan"), -1.0):
        assert clip([ok], max_norm=bad) == mm.MOE_EINVAL
    for bad in (float("nan"), -1.0, 0.0, float("inf")):
        assert clip([ok], unscale=bad) == mm.MOE_EINVAL
    for bad in ((2 * AT, 3 * AT, 100, 2, 0), (2 * AT, 3 * AT, 100, 0, -1), (None, 3 * AT, 100, 0, 0), (2 * AT, None, 100, 0, 0), (2 * AT + 2, 3 * AT, 100, 0, 0),
                (2 * AT, 3 * AT + 1, 100, 1, 1)):
        assert clip([ok, bad]) == mm.MOE_EINVAL, bad
    assert clip([(2 * AT, 3 * AT, 1 << 40, 0, 0)]) == mm.MOE_ESHAPE
    assert clip([(2 * AT, 3 * AT, 1 << 38, 0, 0)]) == mm.MOE_ESHAPE
    assert clip([ok], ws=None) == clip([ok], ws=AT + 16) == clip([ok], ws_bytes=100) == mm.MOE_EWORKSPACE


def test_overlaps_of_clipping():
    """(refused ones only; an empty workspace tells those that would run)"""
    def says(*entries):
        return clip(list(entries), ws=None)
    fine = mm.MOE_EWORKSPACE
    A = 16 * AT
    assert says((A, A, 100, 0, 0)) == says((A, A, 100, 1, 1)) == fine                                  # in place
    assert says((A, A, 100, 0, 1)) == says((A, A, 100, 1, 0)) == mm.MOE_EINVAL                         # of another type
    assert says((A, A + 4, 100, 0, 0)) == says((A + 4, A, 100, 0, 0)) == mm.MOE_EINVAL
    assert says((A, A, 100, 0, 0), (A + 400, A + 400, 5, 0, 0)) == fine                                # neighbours
    assert says((A, A, 101, 0, 0), (A + 400, A + 400, 5, 0, 0)) == mm.MOE_EINVAL
    assert says((A, A, 100, 0, 0), (A, A, 100, 0, 0)) == mm.MOE_EINVAL                                 # the same tensor twice
    assert says((A, 2 * A, 100, 0, 0), (A, 3 * A, 100, 0, 0)) == fine                                  # ... read twice
    assert says((A, 2 * A, 100, 0, 0), (A, 2 * A + 396, 100, 0, 0)) == mm.MOE_EINVAL
    assert says((A, 2 * A, 100, 0, 0), (2 * A + 396, 3 * A, 100, 0, 0)) == mm.MOE_EINVAL               # an out over another's gradient
    assert says((A, 2 * A, 100, 0, 0), (2 * A, A, 100, 0, 0)) == mm.MOE_EINVAL
    assert says((A, A, 100, 0, 0), (A + 40, 2 * A, 10, 0, 0)) == mm.MOE_EINVAL
    assert says((A, 3 * A, 1000, 0, 0), (A + 4, 2 * A, 10, 0, 0), (4 * A, A + 3000, 10, 0, 0)) == mm.MOE_EINVAL
    assert says((A, A, 0, 0, 0), (A, A, 100, 0, 0)) == fine                                            # empty ones overlap nothing


def test_binding_refuses_what_does_not_fit():
    torch = pytest.importorskip("torch")
    t = torch.zeros(4, 4, dtype=torch.float16)
    for call in (lambda: mm.GradList([t], [t, t]), lambda: mm.GradList([t.int()]), lambda: mm.GradList([torch.zeros(4)]), lambda: mm.ExpertGrads([]),
                 lambda: mm.ExpertGrads([(t, t, t)]), lambda: mm.ExpertGrads([(t, t)]), lambda: mm.GradList([t] * 1025)):
        with pytest.raises(mm.MoeError):
            call()


@pytest.mark.skipif(OBJDUMP is None, reason="needs llvm-objdump")
def test_transfers_into_lds_after_lane_reads(tmp_path):
    """A memory instruction needs five wait states after a lane read that wrote its scalar base, and M0 is written by scalar instructions only: the
    compiler does not look after either in front of inline assembly.  And no kernel here spills to memory."""
    transfers = 0
    for i, code in enumerate(_code_objects()):
        if b"train_rows_kernel" not in code and b"train_weights_kernel" not in code:
            continue
        obj = tmp_path / f"{i}.co"
        obj.write_bytes(code)
        asm = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", str(obj)], capture_output=True, text=True, check=True).stdout
        assert "scratch_store" not in asm and "buffer_store" not in asm
        recent = []                                        # the last instructions: (scalars a lane read wrote, wait states)
        for line in asm.splitlines():
            ins = re.match(r"\s+([a-z]\w+)\s*(.*?)\s*(//.*)?$", line)
            if not ins:
                continue
            name, args = ins.group(1), ins.group(2)
            if name.startswith("global_load_lds"):
                transfers += 1
                lo, hi = map(int, re.search(r"s\[(\d+):(\d+)\]", args).groups())
                states = 0
                for wrote, wait in reversed(recent):
                    if states >= 5:
                        break
                    assert not wrote & {lo, hi}, line
                    states += wait
            dst = re.match(r"s(\d+)", args)
            lane = {int(dst.group(1))} if name in ("v_readlane_b32", "v_readfirstlane_b32") and dst else set()
            assert name.startswith("s_") or not args.startswith("m0,"), line
            recent = recent[-8:] + [(lane, 1 + int(args, 0) if name == "s_nop" else 1)]
    assert transfers > 50
