"""e4m3 experts and products with as many rows as the tile kernel takes: results against 64 bits, and what a call leaves in its workspace against the
quantizers."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

from paper_2407_14417_amd import binding as mm
from tests import fp8_ref
from tests.common import assert_ffn_close, unsplit_workspace_bytes
from tests.gpu_common import dev
from tests.test_gpu_fp8 import check_product, normal, on_device, quantized_matrix, rng_of, rows_per_chunk, spoiled, tiles_of

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


# ---------------------------------------------------------------- references in 64 bits on the device

VALUES = torch.from_numpy(fp8_ref.VALUES)


def values(codes, scale, rows):
    """64-bit values of codes [n,c]: scales [ceil(c/128), n] of rows, or [ceil(n/128), ceil(c/128)] of a matrix."""
    v = VALUES.to(codes.device)[codes.long()]
    s = scale.double().t() if rows else scale.double().repeat_interleave(128, 0)[: codes.shape[0]]
    return v * s.repeat_interleave(128, 1)[:, : codes.shape[1]]


def cut_bound(xv, wv):
    total = torch.zeros(xv.shape[0], wv.shape[0], dtype=torch.float64, device=xv.device)
    for c in range(0, xv.shape[1], 8):
        total += 8 * 2.0 ** -13 * (xv[:, None, c:c + 8].abs() * wv[None, :, c:c + 8].abs()).amax(2)
    return total


def check_on_device(y, xv, wv, half, what):
    """Every result within the bounds of fp8_ref.sum_bound and fp8_ref.rounded; fp16 results of some rows within fp8_ref.cut_bound besides (of
    the others: the largest of eight products is at most their sum)."""
    inn = xv.shape[1]
    ref, mag = xv @ wv.t(), xv.abs() @ wv.abs().t()
    bound = (256 + inn / 128 + 16) * 2.0 ** -24 * mag + (ref.abs() * 2.0 ** -11 + 2.0 ** -25 if half else ref.abs() * 2.0 ** -24)
    err = (y.double() - ref).abs()
    assert bool((err <= (bound + 8 * 2.0 ** -13 * mag if half else bound)).all()), what
    if half:
        some = torch.unique(torch.linspace(0, y.shape[0] - 1, 24).long()).to(y.device)
        assert bool((err[some] <= bound[some] + cut_bound(xv[some], wv)).all()), what
    assert float(err.norm()) <= float(ref.norm()) * (2.0 ** -11 + 2.0 ** -13 if half else 2.0 ** -19), what


def generator(*key):
    return torch.Generator(device="cuda").manual_seed(hash(key) % (1 << 31))


def random_half(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).half()


def quantized_rows(x):
    n, inn = x.shape
    codes, scale = torch.empty(n, inn, dtype=torch.uint8, device="cuda"), torch.empty(-(-inn // 128), n, device="cuda")
    mm.moe_quantize_fp8_rows(x, codes, scale)
    return codes, scale


def result(rows, out, half, room=8, shift=0):
    """Rows of NaN for a product, `shift` values off a 16-byte boundary, and the memory around them."""
    whole = torch.full((rows * out + 2 * room + shift,), float("nan"), dtype=torch.float16 if half else torch.float32, device="cuda")
    return whole[room + shift: room + shift + rows * out].view(rows, out), (whole[: room + shift], whole[room + shift + rows * out:])


# ---------------------------------------------------------------- products

@pytest.mark.parametrize("n,inn,out,shift", [(140, 384, 2048, 0), (150, 896, 2080, 1), (300, 1152, 4099, 0), (1488, 1488, 2051, 1), (600, 1040, 4099, 3),
                                             (257, 1424, 6001, 0), (64, 1424, 13001, 0), (1000, 1424, 2049, 1)])
@pytest.mark.parametrize("half", [False, True])
def test_product_of_many_rows(n, inn, out, shift, half):
    """Widths that end inside a block, odd numbers of results, results off 16-byte boundaries."""
    assert rows_per_chunk(n, out, inn, exact=not half) > 0
    print(f"product {n} x {inn} -> {out} half {half}", flush=True)
    g = generator(n, inn, out)
    w, (codes, scale) = mm.quantize_mat_fp8(random_half(g, out, inn, scale=0.02)), quantized_rows(random_half(g, n, inn))
    y, around = result(n, out, half, shift=shift)
    mm.moe_matmul_fp8(w, codes, scale, y)
    check_on_device(y, values(codes, scale, True), values(w.data, w.scale, False), half, (n, inn, out))
    assert all(bool(a.isnan().all()) for a in around)


@pytest.mark.parametrize("inn", [1424, 1536])
@pytest.mark.parametrize("half", [False, True])
def test_stages_come_round_with_every_number_of_tiles(half, inn):
    """Twelve blocks of columns, so that every stage of LDS is filled again several times, with 1 to 16 (fp32 results: 10) tiles of 16 rows in a
    chunk, odd and even; the last block whole and not."""
    out, seen = 13000, set()
    g = generator(inn, half)
    w = mm.quantize_mat_fp8(random_half(g, out, inn, scale=0.02))
    wv = values(w.data, w.scale, False)
    for n in list(range(5, 300, 13)) + list(range(300, 4300, 61)):
        per = rows_per_chunk(n, out, inn, exact=not half)
        tiles = set(tiles_of(n, per)) if per else set()
        if tiles <= seen:
            continue
        seen |= tiles
        print(f"n={n} chunks of {per}: {sorted(tiles)}", flush=True)
        codes, scale = quantized_rows(random_half(g, n, inn))
        y, around = result(n, out, half)
        mm.moe_matmul_fp8(w, codes, scale, y)
        check_on_device(y, values(codes, scale, True), wv, half, n)
        assert all(bool(a.isnan().all()) for a in around)
    assert seen == set(range(1, 17 if half else 11)), seen


@pytest.mark.parametrize("half", [False, True])
def test_every_column_of_many_rows_meets_its_own(half):
    """Row r of x holds one value, at column r: the product is column r of the matrix."""
    n, inn, out = 1488, 1488, 2051
    assert rows_per_chunk(n, out, inn, exact=not half) > 0
    w, (codes, scale) = mm.quantize_mat_fp8(random_half(generator(1), out, inn)), quantized_rows(torch.eye(n, device="cuda").half())
    y, _ = result(n, out, half)
    mm.moe_matmul_fp8(w, codes, scale, y)
    want = values(w.data, w.scale, False).t()
    # one product, two scales: 448/448 and the matrix's, three roundings
    assert bool(((y.double() - want).abs() <= want.abs() * (4 * 2.0 ** -24 + (2.0 ** -11 if half else 0)) + (2.0 ** -25 if half else 0)).all())


@pytest.mark.parametrize("half", [False, True])
def test_scales_of_very_different_size_with_many_rows(half):
    n, inn, out = 150, 896, 2080
    assert rows_per_chunk(n, out, inn, exact=not half) > 0
    g, rng = generator(2), rng_of(32)
    power = lambda lo, hi, *s: torch.from_numpy(2.0 ** rng.integers(lo, hi, s)).cuda().repeat_interleave(128, 1)  # noqa: E731
    x = (random_half(g, n, inn) * power(-9, 10, n, 7)).half()
    w = mm.quantize_mat_fp8((random_half(g, out, inn, scale=0.02) * power(-6, 7, 17, 7).repeat_interleave(128, 0)[:out]).half())
    codes, scale = quantized_rows(x)
    y, _ = result(n, out, half)
    mm.moe_matmul_fp8(w, codes, scale, y)
    assert bool(y.isfinite().all())
    check_on_device(y, values(codes, scale, True), values(w.data, w.scale, False), half, n)


@pytest.mark.parametrize("half", [False, True])
def test_infinities_and_nan_of_many_rows_stay_in_theirs(half):
    n, inn, out = 140, 384, 2048
    assert rows_per_chunk(n, out, inn, exact=not half) > 0
    g = generator(3)
    x, m = random_half(g, n, inn), random_half(g, out, inn, scale=0.02)

    def run(x, m):
        y, _ = result(n, out, half)
        mm.moe_matmul_fp8(mm.quantize_mat_fp8(m), *quantized_rows(x), y)
        return y
    clean = run(x, m)
    assert bool(clean.isfinite().all())
    bad = x.clone()
    bad[n - 1, 200], bad[n // 2, 5], bad[17, 383] = float("inf"), float("nan"), -float("inf")
    y, rows = run(bad, m), torch.tensor([n - 1, n // 2, 17], device="cuda")
    keep = torch.ones(n, dtype=torch.bool, device="cuda")
    keep[rows] = False
    assert bool(y[rows].isnan().all()) and torch.equal(y[keep], clean[keep])
    for poison in (float("nan"), float("inf")):             # a block of the matrix: its 128 results and no others
        mb = m.clone()
        mb[1300, 300] = poison
        y = run(x, mb)
        assert bool(y[:, 1300].isnan().all())
        assert torch.equal(y[:, :1280], clean[:, :1280]) and torch.equal(y[:, 1408:], clean[:, 1408:])


# ---------------------------------------------------------------- grouped products

@pytest.mark.parametrize("T,E,k,inn,out,favour,drop", [(700, 6, 2, 1040, 2051, None, 0), (700, 6, 2, 1040, 4099, 4, 37), (300, 3, 2, 1424, 4099, None, 9),
                                                       (1200, 5, 1, 1296, 4099, None, 0), (900, 32, 8, 1168, 1001, 31, 100), (600, 4, 2, 1424, 6001, None, 1),
                                                       (400, 32, 4, 1168, 2050, 0, 0)])
@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("gather", [True, False])
def test_grouped_product_of_many_rows(T, E, k, inn, out, favour, drop, half, gather):
    """Chunks of several tiles, of experts with many rows, few and none; rows behind the last expert are left as they were."""
    P = T * k
    assert rows_per_chunk(P, out, inn, E, T if gather else P, gather, not half) >= 48
    print(f"grouped T={T} E={E} k={k} {inn} -> {out} half {half} gather {gather}", flush=True)
    rng, g = rng_of(T, E, inn, 33), generator(T, E, inn)
    idx = np.stack([rng.permutation(E - 1 if E > k + 1 else E)[:k] for _ in range(T)])       # (one expert without a row where there are enough)
    if favour is not None:
        idx[:, 0] = favour
    flat = idx.reshape(-1).copy()
    flat[P - drop:] = E
    perm = np.argsort(flat, kind="stable").astype(np.int32)
    off = np.concatenate([[0], np.cumsum(np.bincount(flat, minlength=E + 1)[:E])]).astype(np.int32)
    codes, scale = quantized_rows(random_half(g, T if gather else P, inn))
    ws = [mm.quantize_mat_fp8(random_half(g, out, inn, scale=0.02)) for _ in range(E)]
    y, around = result(P, out, half)
    mm.moe_matmul_fp8_grouped(mm.MatGroup(ws), codes, scale, dev(off), dev(perm) if gather else None, k, y)
    xv = values(codes, scale, True)
    rows = torch.from_numpy(perm).cuda().long() // k if gather else torch.arange(P, device="cuda")
    for e in range(E):
        a, b = int(off[e]), int(off[e + 1])
        if a < b:
            check_on_device(y[a:b], xv[rows[a:b]], values(ws[e].data, ws[e].scale, False), half, f"expert {e}")
    assert bool(y[off[E]:].isnan().all()) and all(bool(a.isnan().all()) for a in around)


@pytest.mark.parametrize("half", [False, True])
@pytest.mark.parametrize("gather", [True, False])
def test_offsets_and_perm_of_many_rows_that_lie_stay_inside(half, gather):
    T, E, inn, out = 700, 4, 528, 4096
    assert rows_per_chunk(T, out, inn, E, T, gather, not half) >= 32
    g = generator(4)
    codes, scale = quantized_rows(random_half(g, T, inn))
    group = mm.MatGroup([mm.quantize_mat_fp8(random_half(g, out, inn, scale=0.02)) for _ in range(E)])
    perm = np.full(T, 3, np.int32)
    perm[:6] = [-5, 1 << 30, T, -1, -(1 << 31), (1 << 31) - 1]
    y, around = result(T, out, half, room=64 * out)
    for off in ([0, -9, 1 << 30, 5, 9], [-100, 300, 200, 100, 1 << 20], [500, 0, 0, 0, 0], [1 << 30] * 5, [0, 700, 0, 700, 0]):
        print(off, flush=True)
        mm.moe_matmul_fp8_grouped(group, codes, scale, dev(np.array(off, dtype=np.int32)), dev(perm) if gather else None, 1, y)
    torch.cuda.synchronize()
    assert all(bool(a.isnan().all()) for a in around)


def behind_work(stream, target, new):
    """On `stream`: a while of work, then `new` copied to `target`.  What runs elsewhere meanwhile sees what was there before."""
    a = torch.ones(4096, 4096, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        for _ in range(60):
            a = torch.mm(a, a).clamp_(-1, 1)
        target.copy_(new)
    a.record_stream(stream)


@pytest.mark.parametrize("T,E,k,inn,out", [(48, 6, 2, 512, 320), (700, 6, 2, 1040, 2051)])
def test_products_on_another_stream_and_in_a_graph(T, E, k, inn, out):
    """The rows come into being on the stream of the call, behind work: a call on another stream would multiply what was there before."""
    g, rng = generator(5, T), rng_of(T, 34)
    idx = np.stack([rng.permutation(E)[:k] for _ in range(T)]).reshape(-1)
    perm, off = dev(np.argsort(idx, kind="stable").astype(np.int32)), dev(np.concatenate([[0], np.cumsum(np.bincount(idx, minlength=E))]).astype(np.int32))
    group = mm.MatGroup([mm.quantize_mat_fp8(random_half(g, out, inn, scale=0.02)) for _ in range(E)])
    x, new = torch.zeros(T, inn, dtype=torch.float16, device="cuda"), [random_half(g, T, inn) for _ in range(4)]
    codes, scale = quantized_rows(x)
    y = torch.empty(T * k, out, device="cuda")

    def step():
        mm.moe_quantize_fp8_rows(x, codes, scale)
        mm.moe_matmul_fp8_grouped(group, codes, scale, off, perm, k, y)
    side = torch.cuda.Stream()
    behind_work(side, x, new[0])
    with torch.cuda.stream(side):
        step()
        got = y.clone()
    side.synchronize()
    torch.cuda.synchronize()
    y.fill_(float("nan"))
    step()
    assert torch.equal(y, got) and bool(y.isfinite().all()) and float(y.abs().max()) > 0
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in new[1:]:
        x.copy_(n)
        graph.replay()
        torch.cuda.synchronize()
        got = y.clone()
        y.fill_(float("nan"))
        step()
        torch.cuda.synchronize()
        assert torch.equal(y, got)


# ---------------------------------------------------------------- hidden rows and blocks

def expert_on_device(g, d, f, scale=0.05):
    return mm.Expert(mm.PREC_FP8B128, *[mm.quantize_mat_fp8(random_half(g, o, i, scale=scale)) for o, i in ((f, d), (f, d), (d, f))])


def routing(layer, x):
    T, E, k = x.shape[0], layer.n_experts, layer.top_k
    new = lambda *s, t=torch.int32: torch.empty(*s, dtype=t, device="cuda")  # noqa: E731
    idx, gate, counts, off, perm = new(T, k), new(T, k, t=torch.float32), new(E), new(E + 1), new(T * k)
    mm.moe_route(layer, x, idx, gate)
    mm.moe_permute(layer, idx, counts, off, perm, mm.alloc_workspace(layer, T))
    return idx, gate, off.tolist(), perm.long()


@pytest.mark.parametrize("T,E,k,d,f", [(700, 6, 2, 128, 1984), (900, 4, 2, 128, 2112), (600, 3, 1, 64, 4032)])
def test_hidden_rows_of_the_tile_kernel_bit_for_bit(T, E, k, d, f):
    """A contraction of one block gives the same sums whichever kernel forms them: the codes and scales that the tile kernel leaves are the quantizer's of
    the fp16 hidden rows that the kernel for few rows leaves."""
    P = T * k
    assert rows_per_chunk(P, f, d, E, T, True, True, True) >= 48 and rows_per_chunk(16, f, d, exact=True, up=True) == 0
    g = generator(T, E, d, f)
    layer = mm.Layer(d, f, k, random_half(g, E, d, scale=0.05), [expert_on_device(g, d, f, 0.3) for _ in range(E)])
    x, ws = random_half(g, T, d), mm.alloc_workspace(layer, T)
    mm.moe_layer_forward(layer, x, torch.empty_like(x), ws)
    _, (h8, hs) = quantized_of(ws, d, f, E, k, T, P, T)
    _, _, off, perm = routing(layer, x)
    small, n = -(-16 // k), 16
    few, y = mm.alloc_workspace(layer, small), torch.empty(n, d, device="cuda")
    at = unsplit_workspace_bytes(d, f, E, k, small) - -(-4 * small * k * d // 256) * 256 - -(-2 * small * k * f // 256) * 256
    seen = 0
    for e in range(E):
        rows = np.unique(np.linspace(off[e], off[e + 1] - 1, 3 * n).astype(int)) if off[e] < off[e + 1] else np.zeros(0, int)
        for i in range(0, len(rows) - n + 1, n):
            some = rows[i:i + n]
            mm.moe_expert_ffn_mixed(layer, e, x[perm[torch.from_numpy(some).cuda()] // k].contiguous(), y, few)
            h = few[at: at + 2 * n * f].view(torch.float16).view(n, f)
            codes, scale = quantized_rows(h.clone())
            assert np.array_equal(h8[some], codes.cpu().numpy()) and np.array_equal(hs[:, some], scale.cpu().numpy()), (e, i)
            seen += n
    assert seen >= 3 * n


def hidden(x, ex):
    """Hidden rows in 64 bits before their rounding, and how far sums of fp32 may bring them off."""
    xv = values(*quantized_rows(x), True)
    a, b = (xv @ values(m.data, m.scale, False).t() for m in (ex.w1, ex.w3))
    da, db = ((256 + x.shape[1] / 128 + 16) * 2.0 ** -24 * (xv.abs() @ values(m.data, m.scale, False).abs().t()) for m in (ex.w1, ex.w3))
    s = a * torch.sigmoid(a)
    # (the derivative of silu is at most 1.1; exponential, quotient and product in 32 bits: a few roundings)
    return s * b, 1.1 * da * b.abs() + s.abs() * db + 1.1 * da * db + 16 * 2.0 ** -24 * (s * b).abs()


@pytest.mark.parametrize("T,E,k,d,f", [(400, 6, 2, 1408, 2816), (500, 5, 3, 1472, 2112), (300, 4, 1, 2048, 3008)])
def test_hidden_rows_of_long_contractions(T, E, k, d, f):
    """Scales are those of the largest hidden value of a block, values are off by half a step of e4m3 and of fp16 and by what sums of fp32 are."""
    P = T * k
    assert rows_per_chunk(P, f, d, E, T, True, True, True) >= 32
    print(f"hidden rows T={T} E={E} k={k} {d} x {f}", flush=True)
    g = generator(T, E, d, f)
    layer = mm.Layer(d, f, k, random_half(g, E, d, scale=0.05), [expert_on_device(g, d, f) for _ in range(E)])
    x, ws = random_half(g, T, d), mm.alloc_workspace(layer, T)
    mm.moe_layer_forward(layer, x, torch.empty_like(x), ws)
    (x8, xs), (h8, hs) = [(dev(c), dev(s)) for c, s in quantized_of(ws, d, f, E, k, T, P, T)]
    codes, scale = quantized_rows(x)
    assert torch.equal(x8, codes) and torch.equal(xs, scale)
    _, _, off, perm = routing(layer, x)
    for e in range(E):
        rows = slice(off[e], off[e + 1])
        if off[e] == off[e + 1]:
            continue
        h, dh = hidden(x[perm[rows] // k].contiguous(), layer.experts[e])
        dh = dh + h.abs() * 2.0 ** -11 + 2.0 ** -25                                   # as fp16
        s = hs[:, rows].t().double().repeat_interleave(128, 1)[:, :f]
        got = values(h8[rows], hs[:, rows], True)
        assert bool(((got - h).abs() <= dh + (h.abs() + dh) * 2.0 ** -4 * (1 + 2.0 ** -20) + s * 2.0 ** -10).all()), e
        pad = -f % 128
        top = lambda v: torch.nn.functional.pad(v, (0, pad)).view(v.shape[0], -1, 128).abs().amax(2)  # noqa: E731
        assert bool(((hs[:, rows].t().double() * 448 - top(h)).abs() <= top(dh) + top(h) * 2.0 ** -23).all()), e


def mixed_layer(g, d, f, E, k):
    """Experts 0, 3 and 5 in e4m3, the others in 4, 8 and 16 bits."""
    experts = []
    for e in range(E):
        mats = [random_half(g, o, i, scale=0.05) for o, i in ((f, d), (f, d), (d, f))]
        kind = {1: (mm.PREC_INT4G64, mm.quantize_mat), 2: (mm.PREC_INT8G64, mm.quantize_mat8), 4: (mm.PREC_FP16, mm.Mat)}.get(e, (mm.PREC_FP8B128, mm.quantize_mat_fp8))
        experts.append(mm.Expert(kind[0], *[kind[1](m) for m in mats]))
    return mm.Layer(d, f, k, random_half(g, E, d, scale=0.05), experts)


def of_parts(layer, x, left_out=()):
    """The block from its experts alone, their rows in 32 bits, averaged in 64."""
    k, (idx, gate, off, perm) = layer.top_k, routing(layer, x)
    out = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    for e in range(layer.n_experts):
        p = perm[off[e]: off[e + 1]]
        if not len(p) or e in left_out:
            continue
        y = torch.empty(len(p), layer.d_model, device="cuda")
        mm.moe_expert_ffn_mixed(layer, e, x[p // k].contiguous(), y, mm.alloc_workspace(layer, len(p)))
        out.index_add_(0, p // k, y.double() * gate.reshape(-1)[p].double()[:, None])
    return out.cpu().numpy()


@pytest.mark.parametrize("T,d,f", [(400, 1408, 2816), (1000, 1408, 1088)])
def test_blocks_of_many_rows_with_experts_of_all_kinds(T, d, f):
    """Experts that run, that another launch runs, that are missing and that come through the swap space, beside each other in the tile kernel."""
    E, k = 6, 2
    assert rows_per_chunk(T * k, f, d, E, T, True, True, True) >= 32 and rows_per_chunk(T * k, d, f, E) >= 32
    g = generator(T, d, f)
    layer = mixed_layer(g, d, f, E, k)
    x = random_half(g, T, d)
    whole, ws = spoiled((T, d), torch.float16), mm.alloc_workspace(layer, T)
    mm.moe_layer_forward(layer, x, whole, ws)
    assert mm.moe_read_status(ws) == 0
    assert_ffn_close(whole.cpu().numpy(), of_parts(layer, x), "block")
    gone, hosts = [], []
    for e, ex in enumerate(layer.experts):
        away = e in (1, 3)
        pin = lambda m: mm.Mat(*[None if t is None else t.cpu().pin_memory() for t in (m.data, m.scale, m.zero)])  # noqa: E731
        hosts.append(mm.Expert(ex.prec, pin(ex.w1), pin(ex.w3), pin(ex.w2), resident=False) if away else None)
        gone.append(mm.Expert(ex.prec, None, None, None, resident=False) if away else ex)
    part, out = mm.Layer(d, f, k, layer.w_gate, gone), spoiled((T, d), torch.float16)
    mm.moe_layer_forward(part, x, out, ws)
    assert mm.moe_read_status(ws) == mm.STATUS_NOT_RESIDENT
    assert_ffn_close(out.cpu().numpy(), of_parts(layer, x, (1, 3)), "block without two experts")
    for slots in (1, 2):
        out = spoiled((T, d), torch.float16)
        assert mm.moe_layer_forward_swap(part, mm.Swap(part, hosts, slots, T), x, out, ws) == 2
        torch.cuda.synchronize()
        assert torch.equal(out, whole)


@pytest.mark.parametrize("T", [1, 2, 130])
def test_block_of_the_mixtral_shape(T):
    d, f, E, k = 4096, 14336, 8, 2
    g = generator(6)
    layer = mm.Layer(d, f, k, random_half(g, E, d, scale=0.02), [expert_on_device(g, d, f, 0.02) for _ in range(E)])
    x, out, ws = random_half(g, T, d), spoiled((T, d), torch.float16), mm.alloc_workspace(layer, T)
    assert T < 130 or (rows_per_chunk(T * k, f, d, E, T, True, True, True) and rows_per_chunk(T * k, d, f, E))
    mm.moe_layer_forward(layer, x, out, ws)
    assert mm.moe_read_status(ws) == 0
    _, gate, off, perm = routing(layer, x)
    want = torch.zeros(T, d, dtype=torch.float64, device="cuda")
    for e, ex in enumerate(layer.experts):
        p = perm[off[e]: off[e + 1]]
        if len(p):
            h = hidden(x[p // k].contiguous(), ex)[0].half()
            y = values(*quantized_rows(h), True) @ values(ex.w2.data, ex.w2.scale, False).t()
            want.index_add_(0, p // k, y * gate.reshape(-1)[p].double()[:, None])
    assert_ffn_close(out.cpu().numpy(), want.cpu().numpy(), f"{T} tokens")


@pytest.mark.parametrize("half", [False, True])
def test_gathered_rows_past_32_bit_offsets(half):
    """Rows of x that lie past 2^32 bytes: the kernel for few rows serves them, however many there are."""
    n, inn, out, E, P = 524_400, 8192, 96, 3, 5000
    assert n * inn > 1 << 32 and rows_per_chunk(P, out, inn, E, n, True, not half) == 0
    g = generator(7)
    codes, scale = torch.zeros(n, inn, dtype=torch.uint8, device="cuda"), torch.zeros(inn // 128, n, device="cuda")
    far = torch.arange(n - 300, n, device="cuda")
    codes[far], scale[:, far] = quantized_rows(random_half(g, 300, inn))
    rows = far[torch.randint(0, 300, (P,), generator=g, device="cuda")]
    rows[::7] = 0
    ws = [mm.quantize_mat_fp8(random_half(g, out, inn, scale=0.02)) for _ in range(E)]
    off = [0, 1700, 1700, P]
    y, around = result(P, out, half)
    mm.moe_matmul_fp8_grouped(mm.MatGroup(ws), codes, scale, dev(np.array(off, dtype=np.int32)), (rows * 2 + 1).int(), 2, y)
    for e in (0, 2):
        at = rows[off[e]: off[e + 1]]
        check_on_device(y[off[e]: off[e + 1]], values(codes[at], scale[:, at].contiguous(), True), values(ws[e].data, ws[e].scale, False), half, e)
    assert all(bool(a.isnan().all()) for a in around)


def test_block_of_more_than_65536_tokens():
    T, d, f, E, k = 70_001, 64, 128, 4, 2
    g = generator(8)
    layer = mm.Layer(d, f, k, random_half(g, E, d, scale=0.2), [expert_on_device(g, d, f, 0.1) for _ in range(E)])
    x, out = random_half(g, T, d), spoiled((T, d), torch.float16)
    ws = mm.alloc_workspace(layer, T)
    mm.moe_layer_forward(layer, x, out, ws)
    assert mm.moe_read_status(ws) == 0
    for lo, hi in ((0, 20_000), (50_000, T)):
        part = spoiled((hi - lo, d), torch.float16)
        mm.moe_layer_forward(layer, x[lo:hi], part, ws)
        assert_ffn_close(out[lo:hi].cpu().numpy(), part.cpu().numpy(), (lo, hi))
