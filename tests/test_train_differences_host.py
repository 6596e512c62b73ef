"""Would the comparison with differences notice a wrong gradient?  The formulas of train_ref, with and without mistakes, on the CPU."""
import pytest

torch = pytest.importorskip("torch")

from tests.train_differences import LIMIT, WHAT, worst
from tests.train_ref import Ref

T, D, F, E, K = 50, 64, 128, 3, 2


@pytest.fixture(scope="module", autouse=True)
def one_thread():
    """(many small products: threads of several test processes would wait for one another)"""
    before = torch.get_num_threads()
    torch.set_num_threads(1)
    yield
    torch.set_num_threads(before)


@pytest.fixture(scope="module")
def block():
    g = torch.Generator().manual_seed(41)
    new = lambda *s, scale=1.0: (torch.randn(*s, generator=g) * scale).half()  # noqa: E731
    w1, w3, w2 = new(E, F, D, scale=D ** -0.5), new(E, F, D, scale=D ** -0.5), new(E, D, F, scale=F ** -0.5)
    x, d_out = new(T, D), new(T, D, scale=0.5)
    key = torch.rand(T, E, generator=g).topk(K, 1).indices.reshape(-1)
    groups = list(torch.sort(key, stable=True).indices.split(torch.bincount(key, minlength=E).tolist()))
    ref = Ref(x, w1, w3, w2, groups, torch.rand(T * K, generator=g).double() + 0.1, K)
    (a, _), (u, _), _ = ref.forward()
    return ref, a.half(), u.half(), d_out


def gradients(block, mistake=""):
    """The formulas by themselves, from the kept rows."""
    ref, a, u, d_out = block
    r = dict(x=torch.zeros(T, D).double(), gate=torch.zeros(T * K).double(), w1=[], w3=[], w2=[])
    at = 0
    for (w1, w3, w2), p in zip(ref.w, ref.groups):
        A, U = a[at: at + len(p)].double(), u[at: at + len(p)].double()
        at += len(p)
        x, do, g = ref.x[p // K], d_out[p // K].double(), ref.g[p][:, None]
        s = torch.sigmoid(A)
        h, q = A * s * U, do @ w2
        slope = s if mistake == "slope" else s * (1 + A * (1 - s))
        da, du = g * q * U * slope, q * A * s * (1.0 if mistake == "gate of d_u" else g)
        if mistake == "columns":
            da[:, :2] = 0
        r["x"].index_add_(0, p // K, da @ w1 + (0 if mistake == "half of d_x" else du @ w3))
        r["gate"][p] = (q * h).sum(1) * (g[:, 0] if mistake == "gate of d_gate" else 1.0)
        r["w1"].append(da.t() @ x)
        r["w3"].append(du.t() @ x)
        r["w2"].append(do.t() @ ((1.0 if mistake == "gate of d_w2" else g) * h))
    r = {k: torch.stack(v) if isinstance(v, list) else v for k, v in r.items()}
    if mistake == "factor":
        r = {k: 0.99 * v for k, v in r.items()}
    if mistake == "expert":
        r = {k: v.index_fill(0, torch.tensor([1]), 0.0) for k, v in r.items()}
    return r


@pytest.mark.parametrize("what", WHAT)
def test_the_right_gradients_fit(block, what):
    grad = gradients(block)[what]
    # (in 64 bits: what is left are the kept rows, rounded to fp16)
    assert worst(block[0], block[3], what, grad, grad) <= LIMIT / 2


@pytest.mark.parametrize("mistake,what", [("slope", "x"), ("slope", "w1"), ("gate of d_u", "x"), ("gate of d_u", "w3"), ("half of d_x", "x"), ("gate of d_gate", "gate"), ("gate of d_w2", "w2"),
                                          ("columns", "w1"), ("expert", "w1"), ("expert", "w3"), ("expert", "w2")] + [("factor", w) for w in WHAT])
def test_wrong_gradients_do_not(block, mistake, what):
    right, wrong = gradients(block)[what], gradients(block, mistake)[what]
    assert worst(block[0], block[3], what, wrong, right) > 2 * LIMIT
    if mistake not in ("columns", "expert"):              # nor where the formula beside it has the same mistake
        assert worst(block[0], block[3], what, wrong, wrong) > 2 * LIMIT
