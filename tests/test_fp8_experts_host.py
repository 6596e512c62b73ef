"""e4m3 experts in the binding: matrices that do not fit their layer are refused before a kernel reads past them.  No kernel is launched here."""
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm

D, F = 320, 704


def mat(out, inn, codes=torch.uint8, scale=torch.float32, shape=None):
    return mm.Mat(torch.zeros(out, inn, dtype=torch.uint8).view(codes), torch.zeros(shape or (-(-out // 128), -(-inn // 128)), dtype=scale))


def layer_with(resident=False, prec=mm.PREC_FP8B128, **mats):
    m = dict(w1=mat(F, D), w3=mat(F, D), w2=mat(D, F)) | mats
    gone = mm.Expert(mm.PREC_FP16, None, None, None, resident=False)
    return mm.Layer(D, F, 1, None, [gone, mm.Expert(prec, m["w1"], m["w3"], m["w2"], resident=resident)])


def refused(code, **k):
    with pytest.raises(mm.MoeError) as e:
        layer_with(**k)
    assert e.value.code == code, e.value


def test_matrices_that_fit():
    layer = layer_with()
    assert layer.n_experts == 2
    layer_with(w1=mat(F, D, torch.float8_e4m3fn))
    refused(mm.MOE_EINVAL, resident=True)                    # not on a GPU
    # another precision is not looked at in this way
    layer_with(prec=mm.PREC_INT8G64, w2=mat(D, F, scale=torch.float16, shape=(D, F // 64)))


@pytest.mark.parametrize("name,out,inn", [("w1", F, D), ("w3", F, D), ("w2", D, F)])
def test_matrices_that_do_not_fit(name, out, inn):
    b, c = -(-out // 128), -(-inn // 128)
    for bad, code in ((mat(inn, out), mm.MOE_ESHAPE), (mat(out - 64, inn), mm.MOE_ESHAPE), (mat(out, inn + 64), mm.MOE_ESHAPE),
                      (mat(out, inn, torch.int8), mm.MOE_EINVAL), (mm.Mat(torch.zeros(out, inn), mat(out, inn).scale), mm.MOE_EINVAL),
                      (mm.Mat(torch.zeros(inn, out, dtype=torch.uint8).t(), mat(out, inn).scale), mm.MOE_EINVAL),
                      (mat(out, inn, scale=torch.float16), mm.MOE_EINVAL), (mat(out, inn, scale=torch.float64), mm.MOE_EINVAL),
                      (mat(out, inn, shape=(b, c - 1)), mm.MOE_ESHAPE), (mat(out, inn, shape=(c, b)), mm.MOE_ESHAPE if b != c else None),
                      (mat(out, inn, shape=(b * c,)), mm.MOE_ESHAPE), (mm.Mat(mat(out, inn).data), mm.MOE_EINVAL),
                      (mm.Mat(mat(out, inn).data, torch.zeros(c, b).t()), mm.MOE_EINVAL)):
        refused(code, **{name: bad})
        refused(code, resident=True, **{name: bad})
    refused(mm.MOE_EINVAL, resident=True, **{name: None})


def test_host_experts_of_a_swap_space():
    layer = layer_with()
    good = mm.Expert(mm.PREC_FP8B128, mat(F, D), mat(F, D), mat(D, F), resident=False)
    for bad, code in ((mat(D, F - 64), mm.MOE_ESHAPE), (mat(D, F, scale=torch.float16), mm.MOE_EINVAL), (mm.Mat(mat(D, F).data), mm.MOE_EINVAL)):
        with pytest.raises(mm.MoeError) as e:
            mm.Swap(layer, [None, mm.Expert(mm.PREC_FP8B128, good.w1, good.w3, bad, resident=False)], 1, 1)
        assert e.value.code == code
