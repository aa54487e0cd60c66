"""The student's layers on the GPU against their definitions in 64 bits (layers_ref.py): types, widths
from one element to long rows, odd sizes and strides, empty and broken rows, far offsets, streams,
captured graphs and autograd."""
import numpy as np
import pytest

torch = pytest.importorskip("torch")

import layers_ref as L
import operators_ref as R
import paper_2405_12491_amd as B
from operators_ref import TYPES, np64

pytestmark = pytest.mark.gpu

inf, nan = float("inf"), float("nan")
NAMES = {torch.float32: "fp32", torch.bfloat16: "bf16", torch.float16: "fp16"}
ids_of = lambda v: NAMES.get(v, str(v))  # noqa: E731


@pytest.fixture(scope="module", autouse=True)
def _cuda():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    B.load_library()
    yield


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(seed, *shape, scale=1.0, dtype=torch.float32):
    return (torch.randn(*shape, generator=_gen(seed), device="cuda") * scale).to(dtype)


def _strided(t, gap, lead=0, fill=None):
    """t's values in a wider buffer: rows `gap` elements further apart, `lead` elements in."""
    n, w = t.shape
    buf = torch.empty(n * (w + gap) + lead + 3, dtype=t.dtype, device=t.device)
    if fill is not None:
        buf.fill_(fill)
    v = buf[lead:lead + n * (w + gap)].view(n, w + gap)[:, :w]
    v.copy_(t)
    return buf, v


def _untouched(buf, view, fill):
    """Every element of buf outside view is still `fill`."""
    probe = buf.clone()
    v = torch.as_strided(probe, view.shape, view.stride(), view.storage_offset())
    v.fill_(fill)
    return bool((probe == fill).all())


def _same_bits(a, b):
    kind = {8: torch.int64, 4: torch.int32, 2: torch.int16, 1: torch.int8}[a.element_size()]
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


WIDTHS = [1, 2, 3, 4, 5, 7, 8, 9, 28, 33, 64, 65, 100, 128, 255, 257, 512, 515, 1000, 2048, 4099]


# ----------------------------------------------------------------------------- embed
def _ids(seed, n, k, nodes, empty=0.1):
    """Ids of k slots with `nodes` entries each (a list), some outside."""
    g = _gen(seed)
    top = torch.tensor(nodes, device="cuda")
    ids = (torch.rand(n, k, generator=g, device="cuda").double() ** 2 * top).long()
    ids = torch.minimum(ids, top - 1)
    out = torch.rand(n, k, generator=g, device="cuda") < empty
    far = torch.randint(0, 3, (n, k), generator=g, device="cuda")
    wrong = torch.where(far == 0, -1, torch.where(far == 1, top.expand(n, k), 2 ** 31 - 1))
    return torch.where(out, wrong, ids).to(torch.int32)


def _check_embed(ids, table, scale, offsets, what=""):
    ref, tol = L.embed(ids, table, scale, offsets)
    out = B.embed(ids, table, scale, offsets)
    R.assert_near(out, ref, tol, table.dtype, f"{what}: embed")
    return out


def _check_embed_grad(ids, grad, entries, scale, offsets, what=""):
    ref, tol = L.embed_grad(ids, grad, entries, scale, offsets)
    out = B.embed_grad(ids, grad, entries, scale, offsets)
    R.assert_near(out, ref, tol, grad.dtype, f"{what}: gradient")
    return out


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", WIDTHS)
def test_embed(width, dtype):
    for n, entries in ((1, 1), (1, 50), (37, 5), (300, 411)):
        ids = _ids(n, n, 1, [entries])
        table = _normal(1, entries, width, dtype=dtype)
        _check_embed(ids, table, 1.0, None, f"{n} {entries}")
        assert _same_bits(B.embed(ids[:, 0], table, 0.3), B.embed(ids, table, 0.3))
        grad = _normal(2, n, width, dtype=dtype)
        _check_embed_grad(ids, grad, entries, 0.3, None, f"{n} {entries}")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [1, 3, 8, 28, 64, 130, 700])
@pytest.mark.parametrize("k", [2, 5, 8, 33, 100])
def test_embed_slots(k, width, dtype):
    """Several slots, each with entries of its own, or all with the same."""
    rng = np.random.default_rng(k)
    nodes = [int(v) for v in rng.integers(1, 40, k)]
    offsets = torch.tensor([0, *np.cumsum(nodes)], device="cuda")
    for n in (1, 3, 70, 900):
        ids = _ids(n, n, k, nodes)
        table = _normal(1, sum(nodes), width, dtype=dtype)
        _check_embed(ids, table, 1.0 / k, offsets, f"{n}")
        _check_embed(ids, table, 1.0 / k, None, f"{n}, one table")
        grad = _normal(2, n, width, dtype=dtype)
        _check_embed_grad(ids, grad, sum(nodes), 1.0 / k, offsets, f"{n}")
        _check_embed_grad(ids, grad, sum(nodes), 1.0 / k, None, f"{n}, one table")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [33, 64, 65, 130, 515, 1024, 2300, 4097])
def test_embed_slots_of_large_tables(width, dtype):
    """Tables past an L2 of 4 MB, and just below, whose rows are split into tiles of 128 to 512 bytes."""
    whole = 2 ** 22 // (width * torch.empty(0, dtype=dtype).element_size())
    for n, entries in ((1, whole + 1), (5, whole), (120, 2 * whole)):
        table = _normal(1, entries, width, dtype=dtype)
        cut = torch.tensor([0, entries // 3, entries // 3, entries // 2, entries], device="cuda")
        ids = _ids(n, n, 4, (cut[1:] - cut[:-1]).clamp(min=1).tolist())
        _check_embed(ids, table, 0.25, cut, f"{n} {entries}")
        buf, view = _strided(table, 3, 1)
        assert _same_bits(B.embed(ids, view, 0.25, cut), B.embed(ids, table, 0.25, cut))


@pytest.mark.parametrize("n", [17, 63, 1000, 1024, 1025, 16_383, 16_384, 16_385])
@pytest.mark.parametrize("sizes", [(1, 0, 1023, 1024, 1025, 511, 512), (0, 0, 5), (200_000, 1, 60_000), (2, 300_000)],
                         ids=str)
def test_embed_grad_sizes_of_slots(sizes, n):
    """Slots of one entry to many, and of none, rows up to where slots are sorted one by one and past it."""
    sizes = list(sizes) * max(1, 1020 // n)
    off = torch.tensor([0, *np.cumsum(sizes)], device="cuda")
    entries = int(off[-1])
    ids = _ids(n, n, len(sizes), [max(v, 1) for v in sizes])
    grad = _normal(2, n, 9)
    _check_embed_grad(ids, grad, entries, 0.5, off, f"{n}")
    # a table that ends inside a slot; ids that lie apart
    short = entries - sizes[-1] // 2
    out = _check_embed_grad(ids, grad, short, 0.5, off, f"{n}, cut")
    _, apart = _strided(ids, 3, 1)
    assert _same_bits(B.embed_grad(apart, grad, short, 0.5, off), out)


@pytest.mark.parametrize("entries", [1, 2, 3, 255, 256, 2046, 2047, 2048, 5000, 300_000, 5_000_000])
def test_embed_grad_numbers_of_entries(entries):
    """One to three passes of the sort, and the numbers where another begins."""
    n = 6000
    g = _gen(entries)
    ids = torch.randint(-1, entries, (n,), generator=g, device="cuda", dtype=torch.int32)
    ids[5:600] = entries - 1
    _check_embed_grad(ids, _normal(1, n, 3), entries, 1.0, None)


@pytest.mark.parametrize("n", [1, 63, 64, 65, 127, 128, 129, 4095, 4096, 4097, 8191, 8193, 20_000, 300_001])
def test_embed_grad_many_rows_of_one_entry(n):
    """Entries with long runs of rows, which begin anywhere: sums of chunks and of many chunks."""
    for lead in (0, 1, 63, 100):
        ids = torch.full((n,), 7, dtype=torch.int32, device="cuda")
        ids[:min(lead, n)] = 3
        if n > 200:
            ids[n // 2:n // 2 + 37] = 9
            ids[-5:] = -1
        _check_embed_grad(ids, _normal(n, n, 20), 12, 1.0, None, f"{lead}")
    ids = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    assert bool((B.embed_grad(ids, _normal(n, n, 20), 12) == 0).all())


def test_embed_grad_order():
    """Sums in an order that the ids decide: equal bits every time, and the sums of two rows rounded
    once."""
    ids = _ids(3, 5000, 1, [900], empty=0.0)[:, 0]
    grad = _normal(4, 5000, 24)
    first = B.embed_grad(ids, grad, 900)
    for _ in range(5):
        assert _same_bits(first, B.embed_grad(ids, grad, 900))
    want = np.zeros((900, 24), np.float32)
    g, at, count = grad.cpu().numpy(), ids.cpu().numpy(), np.bincount(ids.cpu().numpy(), minlength=900)
    for r in range(5000):
        want[at[r]] += g[r]
    few = count <= 2
    assert np.array_equal(first.cpu().numpy()[few], want[few])


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width,gap,lead", [(1, 1, 1), (5, 3, 1), (64, 7, 3), (515, 1, 0)])
def test_embed_strided(width, gap, lead, dtype):
    n, k, entries = 41, 3, 77
    ids = _ids(1, n, k, [entries] * k)
    _, sids = _strided(ids, 2, 1, fill=0)
    table, grad = _normal(2, entries, width, dtype=dtype), _normal(3, n, width, dtype=dtype)
    _, stable = _strided(table, gap, lead, fill=nan)
    _, sgrad = _strided(grad, gap, lead, fill=nan)
    buf, out = _strided(torch.zeros_like(grad), gap, lead, fill=5.0)
    assert B.embed(sids, stable, out=out) is out
    assert _same_bits(out, B.embed(ids, table)) and _untouched(buf, out, 5.0)
    buf, out = _strided(torch.zeros_like(table), gap, lead, fill=5.0)
    assert B.embed_grad(sids, sgrad, entries, out=out) is out
    assert _same_bits(out, B.embed_grad(ids, grad, entries)) and _untouched(buf, out, 5.0)
    # a column of ids
    assert _same_bits(B.embed(sids[:, 1], table), B.embed(ids[:, 1].contiguous(), table))


def test_embed_broken_rows():
    """Infinities and NaN stay with the rows that read them."""
    table = _normal(1, 6, 40)
    table[0], table[1], table[2, 3] = nan, inf, -inf
    ids = torch.tensor([[0, -1], [1, 3], [1, 2], [2, 4], [3, 5], [-1, 6]], dtype=torch.int32, device="cuda")
    out = _check_embed(ids, table, 2.0, None)
    assert bool((out[5] == 0).all()) and bool(torch.isfinite(out[4]).all())
    grad = _normal(2, 6, 40)
    grad[0], grad[2, 7] = nan, inf
    got = _check_embed_grad(ids, grad, 6, 2.0, None)
    assert bool(torch.isfinite(got[3:]).all())


def test_embed_offsets_past_the_table():
    """Slots whose entries lie outside the table are empty, whatever the offsets say."""
    off = torch.tensor([0, 4, -3, 9, 2 ** 62, 20], device="cuda")
    ids = torch.randint(-2, 12, (50, 5), generator=_gen(1), device="cuda", dtype=torch.int32)
    table = _normal(1, 8, 6)
    at = torch.stack([ids[:, 0].long(), ids[:, 1].long() + 4, ids[:, 2].long() - 3], 1)
    ok = torch.zeros(50, 5, dtype=torch.bool, device="cuda")
    ok[:, 0] = (ids[:, 0] >= 0) & (ids[:, 0] < 4)
    want = torch.where(ok[:, :1], table[at[:, 0].clamp(0, 7)], 0.0)
    assert torch.equal(B.embed(ids, table, offsets=off), want)
    grad = B.embed_grad(ids, _normal(2, 50, 6), 8, offsets=off)
    assert bool((grad[4:] == 0).all())


@pytest.mark.parametrize("n", [50, 4000, 17_000])
def test_embed_grad_offsets_past_the_table(n):
    """The same for the gradient, however many pairs are sorted and however: by all of them, by slots, in passes.
    Slots that share no entry may stand in any order."""
    ids = torch.randint(-2, 12, (n, 5), generator=_gen(n), device="cuda", dtype=torch.int32)
    table, grad = _normal(1, 8, 6), _normal(2, n, 6)
    for off in ([0, 4, 4, 9, 30, 2 ** 62], [6, 8, 0, 3, 3, 5]):
        _check_embed(ids, table, 0.5, torch.tensor(off, device="cuda"), f"{off}")
        _check_embed_grad(ids, grad, 8, 0.5, torch.tensor(off, device="cuda"), f"{off}")
    # a slot that begins below 0 is empty
    off, cut = torch.tensor([0, 4, -3, 6, 8, 20], device="cuda"), ids.clone()
    cut[:, 2] = -1
    assert _same_bits(B.embed(ids, table, offsets=off), B.embed(cut, table, offsets=off))
    _check_embed_grad(cut, grad, 8, 0.5, off)
    assert _same_bits(B.embed_grad(ids, grad, 8, 0.5, off), B.embed_grad(cut, grad, 8, 0.5, off))


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [1, 5, 64, 130, 700])
def test_embed_one_entry_at_any_distance(width, dtype):
    """The distance between rows counts for nothing where there is one: a table of one entry, and one row."""
    code = list(NAMES).index(dtype)
    table, grad = _normal(1, 1, width, dtype=dtype), _normal(2, 9, width, dtype=dtype)
    ids = torch.tensor([[0, -1, 0], [-1, -1, -1], [1, 0, 2 ** 31 - 1]] * 3, dtype=torch.int32, device="cuda")
    off = torch.tensor([0, 1, 1, 1], device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    for n, k in ((9, 3), (1, 3), (9, 1)):
        own, g = ids[:n, :k].contiguous(), grad[:n]
        for offsets in (None, off[:k + 1]):
            ref, tol = L.embed(own, table, 1.5, offsets)
            gref, gtol = L.embed_grad(own, g, 1, 1.5, offsets)
            bytes_ = B.bridger_embed_backward_workspace(n, k, 1, width)
            workspace = torch.empty(bytes_, dtype=torch.uint8, device="cuda")
            for ld in (0, -1, width - 1, 10 ** 12, 2 ** 62, -2 ** 62):
                out, got = torch.full((n, width), nan, dtype=dtype, device="cuda"), torch.full_like(table, nan)
                row = [k, width, width] if n > 1 else [ld] * 3
                at = None if offsets is None else offsets.data_ptr()
                B.bridger_embed(own.data_ptr(), row[0], at, table.data_ptr(), ld, code, n, k, 1, width, 1.5,
                                out.data_ptr(), row[1], stream)
                R.assert_near(out, ref, tol, dtype, f"{n} {k} {ld}")
                B.bridger_embed_backward(own.data_ptr(), row[0], at, g.data_ptr(), row[2], code, n, k, 1, width, 1.5,
                                         got.data_ptr(), ld, workspace.data_ptr(), bytes_, stream)
                R.assert_near(got, gref, gtol, dtype, f"{n} {k} {ld}: gradient")


def test_embed_no_rows():
    table = _normal(1, 9, 12)
    none = torch.empty(0, 4, dtype=torch.int32, device="cuda")
    assert B.embed(none, table).shape == (0, 12)
    out = torch.full((9, 12), nan, device="cuda")
    B.embed_grad(none, torch.empty(0, 12, device="cuda"), 9, out=out)
    assert bool((out == 0).all())


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
def test_embed_in_autograd(dtype):
    ids = _ids(1, 60, 3, [20, 30, 7])
    off = torch.tensor([0, 20, 50, 57], device="cuda")
    table = _normal(2, 57, 33, dtype=dtype).requires_grad_()
    out = B.embed(ids, table, 0.5, off)
    assert _same_bits(out.detach(), B.embed(ids, table.detach(), 0.5, off))
    up = _normal(3, 60, 33, dtype=dtype)
    got, = torch.autograd.grad(out, table, up)
    assert _same_bits(got, B.embed_grad(ids, up, 57, 0.5, off))
    B.embed(ids, table, 0.5, off).sum().backward()           # a broadcast gradient
    R.assert_near(table.grad, *L.embed_grad(ids, torch.ones_like(up), 57, 0.5, off), dtype)
    with torch.no_grad():
        assert not B.embed(ids, table).requires_grad
    with pytest.raises(RuntimeError, match="outputs that are given"):
        B.embed(ids, table, out=torch.empty(60, 33, dtype=dtype, device="cuda"))


def test_embed_gradient_against_differences():
    """The sum of out * up, linear in the table: differences are exact up to rounding."""
    ids = _ids(1, 40, 2, [11, 11])
    table, up = _normal(2, 11, 5), _normal(3, 40, 5)
    grad = np64(B.embed_grad(ids, up, 11, 0.7))
    base = np64(B.embed(ids, table, 0.7))
    for e, j in ((0, 0), (3, 2), (10, 4)):
        moved = table.clone()
        moved[e, j] += 1.0
        diff = ((np64(B.embed(ids, moved, 0.7)) - base) * np64(up)).sum()
        # 80 values of out, each off by 3 roundings of at most 8
        assert abs(diff - grad[e, j]) <= 80 * 3 * R.U * 8 * np.abs(np64(up)).max()


# --------------------------------------------------------------------------- dropout
def _seed(a=1234567890123, b=7):
    return torch.tensor([a, b], device="cuda")


def _check_dropout(x, p, seed, residual=None, layer=0, what=""):
    ref, tol = L.dropout(x, p, seed, residual, layer)
    out = B.dropout(x, p, seed, residual, layer)
    R.assert_near(out, ref, tol, x.dtype, f"{what}: dropout")
    return out


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [1, 2, 3, 4, 5, 7, 8, 9, 15, 16, 17, 28, 33, 64, 100, 347, 512, 515, 2047, 4099, 9001])
def test_dropout(width, dtype):
    for n, p, layer in ((1, 0.5, 0), (13, 0.1, 5), (70, 0.3, 2 ** 31 - 1)):
        x, res = _normal(width, n, width, dtype=dtype), _normal(7, n, width, dtype=dtype)
        _check_dropout(x, p, _seed(), None, layer, f"{n}")
        _check_dropout(x, p, _seed(-3, -1), res, layer, f"{n} residual")


def test_dropout_numbers():
    """Every bit of the 32 counts: the choice of two million elements, whose numbers' upper halves
    meet the limit's some thirty times."""
    x = torch.ones(500, 4001, device="cuda")
    for p in (0.1, 0.9, 0.25, 2.0 ** -32, 1 - 2.0 ** -32, 0.3 + 1e-7):
        out = B.dropout(x, p, _seed(), layer=1)
        assert np.array_equal(out.cpu().numpy() != 0, L.kept(500, 4001, p, _seed().tolist(), 1)), p
    assert torch.equal(B.dropout(x, 0.0, _seed()), x)
    assert bool((B.dropout(x, 1.0, _seed()) == 0).all())
    share = float((B.dropout(x, 0.3, _seed()) == 0).float().mean())
    # 2 million independent choices: a standard deviation of 3.3e-4
    assert abs(share - 0.3) < 6 * 3.3e-4
    a = B.dropout(x, 0.5, _seed(1, 2)) != 0
    for other in (B.dropout(x, 0.5, _seed(1, 3)), B.dropout(x, 0.5, _seed(2, 2)),
                  B.dropout(x, 0.5, _seed(1, 2), layer=1), B.dropout(x, 0.5, _seed(1 + 2 ** 32, 2))):
        assert abs(float((a == (other != 0)).float().mean()) - 0.5) < 6 * 3.6e-4


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width,gap,lead", [(1, 1, 1), (5, 3, 1), (64, 7, 3), (515, 1, 0), (5003, 2, 5)])
def test_dropout_strided_and_in_place(width, gap, lead, dtype):
    x, res = _normal(1, 19, width, dtype=dtype), _normal(2, 19, width, dtype=dtype)
    want = B.dropout(x, 0.4, _seed(), res)
    _, sx = _strided(x, gap, lead, fill=nan)
    _, sres = _strided(res, gap + 1, lead, fill=nan)
    buf, out = _strided(torch.zeros_like(x), gap, lead, fill=5.0)
    assert B.dropout(sx, 0.4, _seed(), sres, out=out) is out
    assert _same_bits(out, want) and _untouched(buf, out, 5.0)
    for which in (0, 1):
        bufs = [_strided(t, gap, lead, fill=5.0) for t in (x, res)]
        out = bufs[which][1]
        B.dropout(bufs[0][1], 0.4, _seed(), bufs[1][1], out=out)
        assert _same_bits(out, want) and _untouched(bufs[which][0], out, 5.0)


def test_dropout_broken_elements():
    """A dropped element is zero, whatever it was."""
    x = torch.full((40, 50), nan, device="cuda")
    x[::2] = inf
    out = B.dropout(x, 0.5, _seed())
    keep = torch.from_numpy(L.kept(40, 50, 0.5, _seed().tolist(), 0)).cuda()
    assert bool((out[~keep] == 0).all()) and not bool(torch.isfinite(out[keep]).any())
    assert bool((B.dropout(x, 1.0, _seed()) == 0).all())
    assert B.dropout(torch.empty(0, 5, device="cuda"), 0.5, _seed()).shape == (0, 5)


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
def test_dropout_in_autograd(dtype):
    x = _normal(1, 30, 37, dtype=dtype).requires_grad_()
    res = _normal(2, 30, 37, dtype=dtype).requires_grad_()
    up = _normal(3, 30, 37, dtype=dtype)
    seed = _seed()
    out = B.dropout(x, 0.3, seed, res, layer=4)
    assert _same_bits(out.detach(), B.dropout(x.detach(), 0.3, seed, res.detach(), 4))
    dx, dres = torch.autograd.grad(out, (x, res), up)
    assert _same_bits(dx, B.dropout(up, 0.3, seed, layer=4)) and torch.equal(dres, up)
    R.assert_near(dx, *L.dropout(up, 0.3, seed, None, 4), dtype)
    only = B.dropout(x.detach(), 0.3, seed, res)
    only.sum().backward()
    assert torch.equal(res.grad, torch.ones_like(up)) and x.grad is None
    out = B.dropout(x, 0.3, seed)
    seed[1] += 1                                   # the next step's numbers before the gradient
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


# ------------------------------------------------------------------------ layer_norm
LN_WIDTHS = [1, 2, 3, 4, 7, 8, 9, 16, 28, 31, 32, 33, 63, 64, 65, 100, 128, 255, 257, 512, 513, 784, 1023, 1025,
             2047, 2049, 4096, 5001, 8192, 8195, 16384, 16389, 32768, 32771]


def _norm_inputs(seed, n, w, dtype, shift=0.5):
    return ((_normal(seed, n, w) * 2 + shift).to(dtype), _normal(seed + 1, n, w, dtype=dtype),
            (1 + _normal(seed + 2, w) * 0.3).to(dtype), _normal(seed + 3, w, scale=0.2, dtype=dtype))


def _check_norm(x, res, w, b, eps=1e-5, what=""):
    """Forward, and the gradients through layer_norm_grad."""
    n, f = x.shape
    stats = torch.full((n, 3), nan, device="cuda")
    y, total = B.layer_norm(x, w, b, residual=res, eps=eps, stats=stats)
    t = x
    if res is not None:
        t = (x.float() + res.float()).to(x.dtype)
        assert _same_bits(t, total), f"{what}: total"
    else:
        assert total is None
    R.assert_near(y, *L.layer_norm(t, w, b, eps), x.dtype, f"{what}: norm")
    g, gt = _normal(9, n, f, dtype=x.dtype), None if res is None else _normal(8, n, f, dtype=x.dtype)
    got = B.layer_norm_grad(g, t, stats, w, grad_total=gt)
    for name, v, ref, tol in zip(("dx", "dweight", "dbias"), got, *L.layer_norm_grad(g, t, w, gt, eps)):
        R.assert_near(v, ref, tol, x.dtype, f"{what}: {name}")
    return y, stats


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", LN_WIDTHS)
def test_layer_norm(width, dtype):
    for n in (1, 5, 70) if width < 1000 else (3,):
        x, res, w, b = _norm_inputs(width, n, width, dtype)
        _check_norm(x, None, w, b, what=f"{n}")
        _check_norm(x, res, w, b, what=f"{n} residual")
    _check_norm(x, None, None, None, what="plain")
    _check_norm(x, res, w, None, what="no bias")
    _check_norm(x, None, None, b, what="no weight")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [40_000, 65_537, 100_003])
def test_layer_norm_long_rows(width, dtype):
    x, res, w, b = _norm_inputs(width, 6, width, dtype)
    _check_norm(x, res, w, b)
    _check_norm(x, None, None, None)


@pytest.mark.parametrize("n", [2, 63, 64, 65, 1023, 1025, 5000, 40_001])
@pytest.mark.parametrize("width", [3, 28, 130])
def test_layer_norm_rows(n, width):
    x, res, w, b = _norm_inputs(n, n, width, torch.float32)
    _check_norm(x, res, w, b)


@pytest.mark.parametrize("width", [28, 700, 5000, 30_000, 70_000])
def test_layer_norm_far_from_zero(width):
    """A mean that a float does not hold to the last bit of the row's spread."""
    x = (_normal(1, 6, width).double() * 2.0 ** -8 + torch.tensor(
        [1000.3, -1000.1, 1e5, 3.7, 0.0, 77.7], device="cuda")[:, None]).float()
    _check_norm(x, None, None, None, eps=1e-9)


@pytest.mark.parametrize("eps", [1e-5, 1e-12])
@pytest.mark.parametrize("width", [28, 1023, 4099, 8001, 13_001, 16_001])
def test_layer_norm_far_rows_of_nearly_equal_elements(width, eps):
    """Rows whose sum in float misses the mean by more than their spread: a few elements one step above the
    others."""
    rng = np.random.default_rng(width)
    first = np.array([12552103.544, 1814612.83, 843109.795, 259470249.0, 7512806.0, 1794.0023, -3.3e8, 77.7], np.float32)
    share = np.array([0.01, 0.001, 0.5])
    step = np.spacing(np.abs(first))
    x = np.concatenate([first[:, None] + step[:, None] * (rng.random((8, width)) < p) for p in share]).astype(np.float32)
    assert np.all((x == np.tile(first, 3)[:, None]) | (x == np.tile(first + step, 3)[:, None]))
    _check_norm(torch.from_numpy(x).cuda(), None, None, None, eps=eps)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids_of)
@pytest.mark.parametrize("width", [3, 5, 28, 700, 9000, 70_000])
def test_layer_norm_extremes(width, dtype):
    """Rows whose squares or sums leave float, and tiny ones."""
    base = _normal(1, 7, width)
    scale = torch.tensor([1e30, 1e-30, 1e19, 1e-19, 3e36, 1e15, 1.0], device="cuda")[:, None]
    x = (base * scale).to(dtype)
    for eps in (0.0, 1e-5):
        y, _ = B.layer_norm(x, eps=eps)
        R.assert_near(y, *L.layer_norm(x, None, None, eps), dtype, f"{eps}")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [1, 3, 28, 700, 9000, 70_000])
def test_layer_norm_equal_and_broken_rows(width, dtype):
    x, res, w, b = _norm_inputs(1, 8, width, dtype)
    x[0] = 0.0
    x[1] = 3.0
    x[2, 0] = nan
    x[3, -1] = inf
    x[4, 0] = -inf
    y, stats = B.layer_norm(x, w, b)[0], None
    R.assert_near(y, *L.layer_norm(x, w, b), dtype)
    assert _same_bits(y[0], b) and _same_bits(y[1], b)
    assert bool(torch.isnan(y[2:5]).all()) and bool(torch.isfinite(y[5:]).all())
    assert bool(torch.isnan(B.layer_norm(x, w, b, eps=0.0)[0][:2]).all())
    # a broken row's gradient stays in its row (and in the weight's)
    stats = torch.empty(8, 3, device="cuda")
    B.layer_norm(x, w, b, stats=stats)
    g = _normal(5, 8, width, dtype=dtype)
    dx, dw, db = B.layer_norm_grad(g, x, stats, w)
    (rx, _, rb), (tx, _, tb) = L.layer_norm_grad(g, x, w)
    R.assert_near(dx[5:], rx[5:], tx[5:], dtype)
    assert bool(torch.isnan(dx[2:5]).all()) and bool(torch.isnan(dw).all())
    R.assert_near(db, rb, tb, dtype)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids_of)
@pytest.mark.parametrize("width", [1, 3, 5, 28, 32, 100, 700, 1030, 4100, 9000, 40_000, 70_001])
def test_layer_norm_grad_of_equal_rows(width, dtype):
    """Rows of one value have a finite gradient, factor (s - mean(s)), however large the value is: what stands
    past a row's end takes no part in it."""
    low = float(torch.finfo(dtype).min)
    for residual in (False, True):
        x = torch.tensor([1e37, 3e36, -2.0 ** 120, low / 2, low, 3.0, 0.0], device="cuda")[:, None].expand(7, width).to(dtype)
        x = x.contiguous()
        _, _, w, b = _norm_inputs(1, 7, width, dtype)
        res = torch.zeros_like(x) if residual else None
        _check_norm(x, res, w, b)
        _check_norm(x, res, None, None)
        stats = torch.empty(7, 3, device="cuda")
        B.layer_norm(x, w, b, stats=stats)
        assert all(bool(torch.isfinite(v).all()) for v in B.layer_norm_grad(_normal(2, 7, width, dtype=dtype), x, stats, w))


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width,gap,lead", [(1, 1, 1), (5, 3, 1), (64, 7, 3), (515, 1, 0), (5003, 2, 5), (70_001, 3, 1)])
def test_layer_norm_strided_and_in_place(width, gap, lead, dtype):
    n = 11
    x, res, w, b = _norm_inputs(1, n, width, dtype)
    stats = torch.empty(n, 3, device="cuda")
    y, total = B.layer_norm(x, w, b, residual=res, stats=stats)
    _, sx = _strided(x, gap, lead, fill=nan)
    _, sres = _strided(res, gap + 1, lead, fill=nan)
    buf, out = _strided(torch.zeros_like(x), gap, lead, fill=5.0)
    tbuf, tout = _strided(torch.zeros_like(x), gap, lead, fill=5.0)
    got = B.layer_norm(sx, w, b, residual=sres, out=out, total=tout)
    assert got[0] is out and got[1] is tout
    assert _same_bits(out, y) and _same_bits(tout, total)
    assert _untouched(buf, out, 5.0) and _untouched(tbuf, tout, 5.0)
    for which in (0, 1):
        bufs = [_strided(t, gap, lead, fill=5.0) for t in (x, res)]
        got, _ = B.layer_norm(bufs[0][1], w, b, residual=bufs[1][1], total=bufs[which][1])
        assert _same_bits(got, y) and _same_bits(bufs[which][1], total)
        assert _untouched(bufs[which][0], bufs[which][1], 5.0)
    alone = torch.zeros_like(x)
    assert _same_bits(B.layer_norm(x, total=alone)[0], B.layer_norm(x)[0]) and _same_bits(alone, x)
    g, gt = _normal(4, n, width, dtype=dtype), _normal(5, n, width, dtype=dtype)
    want = B.layer_norm_grad(g, total, stats, w, grad_total=gt)
    _, sg = _strided(g, gap, lead, fill=nan)
    _, sgt = _strided(gt, gap + 2, lead, fill=nan)
    buf, out = _strided(torch.zeros_like(x), gap, lead, fill=5.0)
    got = B.layer_norm_grad(sg, tout, stats, w, grad_total=sgt, out=out)
    assert got[0] is out and _untouched(buf, out, 5.0)
    assert all(_same_bits(a, v) for a, v in zip(got, want))
    dx, dw, db = B.layer_norm_grad(g, total, stats, w, grad_total=gt, weights=False)
    assert _same_bits(dx, want[0]) and dw is None and db is None


def test_layer_norm_no_rows():
    x, w = torch.empty(0, 12, device="cuda"), torch.ones(12, device="cuda")
    y, total = B.layer_norm(x, w, residual=x)
    assert y.shape == total.shape == (0, 12)
    dx, dw, db = B.layer_norm_grad(x, x, torch.empty(0, 3, device="cuda"), w)
    assert dx.shape == (0, 12) and bool((dw == 0).all()) and bool((db == 0).all())


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
def test_layer_norm_in_autograd(dtype):
    x, res, w, b = (t.requires_grad_() for t in _norm_inputs(1, 30, 37, dtype))
    g, gt = _normal(3, 30, 37, dtype=dtype), _normal(4, 30, 37, dtype=dtype)
    stats = torch.empty(30, 3, device="cuda")
    with torch.no_grad():
        y, total = B.layer_norm(x, w, b, residual=res, stats=stats)
        want = B.layer_norm_grad(g, total, stats, w, grad_total=gt)
    out = B.layer_norm(x, w, b, residual=res)
    assert _same_bits(out[0].detach(), y) and _same_bits(out[1].detach(), total)
    got = torch.autograd.grad(out, (x, res, w, b), (g, gt))
    assert all(_same_bits(a, v) for a, v in zip(got, (want[0], want[0], *want[1:])))
    # only one of the outputs, and only some of the leaves
    y, _ = B.layer_norm(x, w, b, residual=res)
    one = torch.autograd.grad(y, (x, w), g)
    with torch.no_grad():
        two = B.layer_norm_grad(g, total, stats, w)
    assert _same_bits(one[0], two[0]) and _same_bits(one[1], two[1])
    _, t = B.layer_norm(x, w, b, residual=res)
    dx, dw, db = torch.autograd.grad(t, (x, w, b), gt)
    assert torch.equal(dx, gt) and bool((dw == 0).all()) and bool((db == 0).all())
    y, none = B.layer_norm(x.detach(), w)
    assert none is None
    dw, = torch.autograd.grad(y.sum(), w)
    with torch.no_grad():
        B.layer_norm(x, w, stats=stats)
        assert _same_bits(dw, B.layer_norm_grad(torch.ones_like(g), x, stats, w)[1])
    loss = (B.layer_norm(x, w, b, residual=res)[0].float() ** 2).sum()
    loss.backward()
    assert x.grad.data_ptr() != res.grad.data_ptr() and torch.equal(x.grad, res.grad)


def test_layer_norm_gradient_against_differences():
    """Central differences of the sum of norm * up in double, from the definition, at inputs moved by
    2^-10: off by the third derivative (under 8 per unit here) times 2^-20 / 6."""
    x, _, w, b = _norm_inputs(5, 4, 9, torch.float32)
    up = _normal(6, 4, 9)
    stats = torch.empty(4, 3, device="cuda")
    y, _ = B.layer_norm(x, w, b, stats=stats)
    dx, dw, db = (np64(v) for v in B.layer_norm_grad(up, x, stats, w))

    def value(x, w, b):
        c = x - x.mean(1, keepdims=True)
        return ((c / np.sqrt((c * c).mean(1, keepdims=True) + 1e-5) * w + b) * np64(up)).sum()

    at, step = [np64(x), np64(w), np64(b)], 2.0 ** -10
    for k, grad in ((0, dx), (1, dw), (2, db)):
        for place in np.ndindex(grad.shape):
            hi, lo = [v.copy() for v in at], [v.copy() for v in at]
            hi[k][place] += step
            lo[k][place] -= step
            diff = (value(*hi) - value(*lo)) / (2 * step)
            assert abs(diff - grad[place]) <= 8 * 2.0 ** -20 / 6 * 40 + 1e-5, (k, place)


@pytest.mark.parametrize("call", ["dropout", "layer_norm", "embed"])
def test_layers_are_differentiated_once(call):
    x = _normal(1, 6, 8).requires_grad_()
    out = {"dropout": lambda: B.dropout(x, 0.5, _seed()), "layer_norm": lambda: B.layer_norm(x)[0],
           "embed": lambda: B.embed(torch.zeros(3, dtype=torch.int32, device="cuda"), x)}[call]()
    grad, = torch.autograd.grad(out.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        grad.sum().backward()


def test_forward_mode():
    """No call gives up a tangent without a word: those that have gradients refuse it."""
    import torch.autograd.forward_ad as fa
    x, res, w, b = _norm_inputs(1, 6, 40, torch.float32)
    ids, seed, one = torch.zeros(3, dtype=torch.int32, device="cuda"), _seed(), torch.ones(6, 40, device="cuda")
    plain = [B.embed(ids, x), B.dropout(x, 0.5, seed), B.layer_norm(x, w, b, residual=res)[0]]
    with fa.dual_level():
        # beside other work in forward mode
        same = [B.embed(ids, x), B.dropout(x, 0.5, seed), B.layer_norm(x, w, b, residual=res)[0]]
        assert all(_same_bits(p, q) for p, q in zip(plain, same))
        for leaf in (x, x.clone().requires_grad_()):
            d = fa.make_dual(leaf, one)
            for call in (lambda: B.embed(ids, d), lambda: B.dropout(d, 0.5, seed), lambda: B.dropout(x, 0.5, seed, d),
                         lambda: B.layer_norm(d, w, b), lambda: B.layer_norm(x, w, b, residual=d)):
                with pytest.raises(NotImplementedError):
                    call()
    for f in (lambda t: B.embed(ids, t), lambda t: B.dropout(t, 0.5, seed), lambda t: B.layer_norm(t)[0]):
        with pytest.raises(RuntimeError):
            torch.func.jvp(f, (x,), (one,))
        with pytest.raises(RuntimeError):
            torch.func.grad(lambda t: f(t).sum())(x)


# ------------------------------------------------------------- together, streams, graphs
def _every(seed=0, n=65, c=1030):
    """name -> (inputs that a replay may scale, call): each operator without autograd."""
    ids = _ids(seed, n, 6, [70] * 6)
    off = torch.arange(0, 421, 70, device="cuda")
    one = _ids(seed + 1, 40 * n, 1, [300])[:, 0]
    table, grad = _normal(seed + 1, 420, c, dtype=torch.bfloat16), _normal(seed + 2, n, c, dtype=torch.float16)
    tall = _normal(seed + 3, 40 * n, 24)
    x, res, w, b = _norm_inputs(seed + 4, n, c, torch.bfloat16)
    stats = torch.empty(n, 3, device="cuda")
    B.layer_norm(x, w, b, stats=stats)
    seeds = _seed(seed, 5)
    z, u = _normal(seed + 9, n, c, scale=3), torch.rand(n, device="cuda", generator=_gen(seed))
    return {
        "embed": ([table], lambda: (B.embed(ids, table, 0.5, off),)),
        "embed_grad": ([grad], lambda: (B.embed_grad(ids, grad, 420, 0.5, off),)),
        "embed_grad_many": ([tall], lambda: (B.embed_grad(one, tall, 300),)),
        "dropout": ([x, res], lambda: (B.dropout(x, 0.3, seeds, res),)),
        "layer_norm": ([x, res], lambda: B.layer_norm(x, w, b, residual=res)),
        "layer_norm_grad": ([grad, w], lambda: B.layer_norm_grad(grad.bfloat16(), x, stats, w)),
        "sample": ([z], lambda: B.sample(z, u, temperature=0.8, top_k=40, top_p=0.9)),
        "sample_all": ([z], lambda: B.sample(z, u, top_p=0.99, temperature=3.0)),
    }


NAMES_ALL = ["embed", "embed_grad", "embed_grad_many", "dropout", "layer_norm", "layer_norm_grad", "sample", "sample_all"]


@pytest.mark.parametrize("name", NAMES_ALL)
@pytest.mark.parametrize("n", [1, 65, 700])
def test_equal_bits_again(name, n):
    call = _every(n=n)[name][1]
    first = [v.clone() for v in call()]
    for _ in range(5):
        assert all(_same_bits(x, y) for x, y in zip(first, call()))


@pytest.mark.parametrize("name", NAMES_ALL)
def test_in_a_graph(name):
    """Captured once, replayed with other inputs in place and eager work between the replays."""
    inputs, call = _every(n=130)[name]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        call()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = call()
    for rep in range(4):
        for v in inputs:
            v.mul_(0.5 + 0.3 * rep)
        torch.cuda.synchronize()
        for v in out:
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        eager = call()
        torch.cuda.synchronize()
        assert all(_same_bits(x, y) for x, y in zip(out, eager)), rep


@pytest.mark.parametrize("n", [600, 30_000])
def test_ids_that_change_between_replays(n):
    """The gradient's plan depends on sizes alone: a graph serves any ids."""
    ids = torch.zeros(n, dtype=torch.int32, device="cuda")
    grad = _normal(1, n, 40)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.embed_grad(ids, grad, 90)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = B.embed_grad(ids, grad, 90)
    for seed in range(4):
        ids.copy_(_ids(seed, n, 1, [[90], [3], [1], [2000]][seed])[:, 0])
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        R.assert_near(out, *L.embed_grad(ids, grad, 90), torch.float32)
        assert _same_bits(out, B.embed_grad(ids, grad, 90))


def test_a_captured_step_draws_anew():
    """seed[1] advances inside the graph: every replay drops other elements."""
    x, seed = torch.ones(50, 70, device="cuda"), _seed(3, 0)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.dropout(x, 0.5, seed)
        seed.add_(torch.tensor([0, 0], device="cuda"))
    s.synchronize()
    step = torch.tensor([0, 1], device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = B.dropout(x, 0.5, seed)
        back = B.dropout(out, 0.5, seed)
        seed.add_(step)
    for rep in range(4):
        g.replay()
        torch.cuda.synchronize()
        keep = torch.from_numpy(L.kept(50, 70, 0.5, (3, rep), 0)).cuda()
        assert torch.equal(out != 0, keep) and torch.equal(back != 0, keep)


def test_two_graphs_and_two_streams_side_by_side():
    """Workspaces are a call's own: graphs and streams that run at once give what each gives alone."""
    ops = [_every(seed=k, n=400) for k in (0, 50)]
    alone = [{k: [v.clone() for v in o[k][1]()] for k in NAMES_ALL} for o in ops]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in ops]
    graphs, outs = [], []
    for s, o in zip(streams, ops):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            for k in NAMES_ALL:
                o[k][1]()
        s.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            outs.append({k: o[k][1]() for k in NAMES_ALL})
        graphs.append(g)
    for _ in range(10):
        for s, g in zip(streams, graphs):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for a, o in zip(alone, outs):
        assert all(_same_bits(x, y) for k in NAMES_ALL for x, y in zip(a[k], o[k]))
    for _ in range(10):
        eager = []
        for s, o in zip(streams, ops):
            with torch.cuda.stream(s):
                eager.append({k: o[k][1]() for k in NAMES_ALL})
    torch.cuda.synchronize()
    for a, o in zip(alone, eager):
        assert all(_same_bits(x, y) for k in NAMES_ALL for x, y in zip(a[k], o[k]))


def test_calls_from_several_threads():
    from concurrent.futures import ThreadPoolExecutor
    ops = [_every(seed=k, n=300) for k in (0, 50, 100)]
    alone = [{k: [v.clone() for v in o[k][1]()] for k in NAMES_ALL} for o in ops]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(10):
                outs = {k: ops[i][k][1]() for k in NAMES_ALL}
            torch.cuda.current_stream().synchronize()
        return all(_same_bits(x, y) for k in NAMES_ALL for x, y in zip(alone[i][k], outs[k]))

    with ThreadPoolExecutor(3) as pool:
        assert all(pool.map(work, range(3)))


def test_with_a_gradient_they_are_refused_in_a_graph():
    x = _normal(1, 6, 8).requires_grad_()
    ids = torch.zeros(3, dtype=torch.int32, device="cuda")
    calls = [lambda: B.embed(ids, x), lambda: B.dropout(x, 0.5, seed), lambda: B.layer_norm(x)[0],
             lambda: B.layer_norm(x.detach(), x[0])[0], lambda: B.dropout(x.detach(), 0.5, seed, x)]
    seed = _seed()
    w = x[0].detach()
    eager = [c() for c in calls]
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        for c in calls[:3] + calls[4:]:
            with pytest.raises(RuntimeError, match="being captured"):
                c()
        with torch.no_grad():
            out = [c() for c in calls]
    for _ in range(3):
        for v in out:
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, e.detach()) for a, e in zip(out, eager))
    sum(e.sum() for e in eager).backward()
    assert bool(torch.isfinite(x.grad).all()) and w.shape == (8,)


def test_a_step_in_a_graph_beside_an_eager_one():
    """embed -> dropout -> layer_norm and back without autograd is captured while an eager graph of the
    same leaves is alive."""
    table = _normal(1, 50, 64).requires_grad_()
    w, b = _normal(2, 64).requires_grad_(), _normal(3, 64).requires_grad_()
    ids, seed, up = _ids(4, 90, 1, [50])[:, 0], _seed(), _normal(5, 90, 64)

    def step():
        with torch.no_grad():
            stats = torch.empty(90, 3, device="cuda")
            h = B.dropout(B.embed(ids, table, 8.0), 0.2, seed)
            y, _ = B.layer_norm(h, w, b, stats=stats)
            dx, dw, db = B.layer_norm_grad(up, h, stats, w)
            return y, B.embed_grad(ids, B.dropout(dx, 0.2, seed), 50, 8.0), dw, db

    eager, _ = B.layer_norm(B.dropout(B.embed(ids, table, 8.0), 0.2, seed), w, b)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        step()
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        out = step()
    for _ in range(3):
        for v in out:
            v.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert _same_bits(out[0], eager.detach())
    grads = torch.autograd.grad(eager, (table, w, b), up)
    assert all(_same_bits(a, v) for a, v in zip(out[1:], grads))


def test_on_another_stream_and_with_torch_between():
    """Outputs are ready for torch on the stream of the call."""
    s = torch.cuda.Stream()
    ops = _every(n=200)
    alone = {k: [v.clone() for v in ops[k][1]()] for k in NAMES_ALL}
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        busy = torch.randn(4096, 4096, device="cuda")
        for _ in range(10):
            busy = busy @ busy * 1e-3
        outs = {k: [v + 0 for v in ops[k][1]()] for k in NAMES_ALL}
    s.synchronize()
    assert all(torch.equal(x, y) for k in NAMES_ALL for x, y in zip(alone[k], outs[k]))


def test_together_with_a_forest():
    """A student of a forest's leaves: predict_leaves -> embed -> dropout -> layer_norm -> class scores, the
    forest's largest scores to learn from, an answer drawn at last."""
    from synth import make_workload
    w = make_workload("rf_d8", 500)
    X = torch.from_numpy(w.X()).cuda()
    off = torch.from_numpy(np.ascontiguousarray(w.forest.tree_offsets)).cuda()
    nodes, k, width, classes = int(off[-1]), len(off) - 1, 48, 10
    with B.Forest(w.forest) as f:
        leaves = f.predict_leaves(X)
    table = _normal(1, nodes, width, scale=0.3).requires_grad_()
    gain, shift = torch.ones(width, device="cuda").requires_grad_(), torch.zeros(width, device="cuda").requires_grad_()
    head = _normal(2, width, classes, scale=0.2).requires_grad_()
    teacher_ids = torch.stack([torch.arange(2, dtype=torch.int32)] * 500).cuda()
    teacher = _normal(3, 500, 2)
    seed = _seed()

    def forward():
        h = B.dropout(B.embed(leaves, table, 1.0 / k, off), 0.1, seed, layer=2)
        y, total = B.layer_norm(h, gain, shift, residual=h)
        return y, total, y @ head

    y, total, logits = forward()
    loss = B.distill_loss(logits, teacher_ids, teacher).sum()
    grads = torch.autograd.grad(loss, (table, gain, shift, head))
    # the same in torch, 64 bits
    ref = [t.detach().double().requires_grad_() for t in (table, gain, shift, head)]
    at = (leaves.long() + off[:-1]).reshape(-1)
    e = ref[0][at].view(500, k, width).sum(1) / k
    keep = torch.from_numpy(L.kept(500, width, 0.1, seed.tolist(), 2)).cuda()
    h = torch.where(keep, e / 0.9, 0.0)
    t = h + h
    c = t - t.mean(1, keepdim=True)
    z = (c / (c.pow(2).mean(1, keepdim=True) + 1e-5).sqrt() * ref[1] + ref[2]) @ ref[3]
    p = torch.softmax(teacher.double(), 1)
    want = -(p * torch.log_softmax(z, 1)[:, :2]).sum() + (p * p.log()).sum()
    # Sums of 100 leaves, 48 features, 10 classes and 500 rows, one after the other: under 1000 roundings
    # of terms that are at most 10 times their sum.
    assert abs(float(loss.detach()) - float(want.detach())) <= 1e4 * R.U * float(want.detach())
    for got, r in zip(grads, torch.autograd.grad(want, ref)):
        assert float((got.double() - r).abs().max()) <= 1e4 * R.U * float(r.abs().max())
    ids, logp = B.sample(logits.detach(), torch.rand(500, device="cuda", generator=_gen(9)), top_k=5)
    _, top = B.top_k(logits.detach(), 5)
    assert bool((top == ids[:, None]).any(1).all()) and bool((logp <= 0).all())


# -------------------------------------------------------------------- sizes and refusals
def test_far_offsets():
    """Rows whose offsets pass 2^31 elements (and 2^32 bytes)."""
    far, c = (1 << 31) + 24, 1000
    buf = torch.empty(2 * far + c, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(buf, (3, c), (far, 1))
    x = _normal(1, 3, c, dtype=torch.bfloat16)
    rows.copy_(x)
    ids = torch.tensor([2, 0, 1, 2, -1], dtype=torch.int32, device="cuda")
    bag = torch.tensor([[2, 0], [1, 2]], dtype=torch.int32, device="cuda")
    assert _same_bits(B.embed(ids, rows), B.embed(ids, x)) and _same_bits(B.embed(bag, rows), B.embed(bag, x))
    assert _same_bits(B.embed_grad(ids[:3], rows, 9), B.embed_grad(ids[:3], x, 9))
    assert _same_bits(B.dropout(rows, 0.5, _seed(), rows), B.dropout(x, 0.5, _seed(), x))
    stats = torch.empty(3, 3, device="cuda")
    assert _same_bits(B.layer_norm(rows, stats=stats)[0], B.layer_norm(x)[0])
    for a, v in zip(B.layer_norm_grad(rows, rows, stats), B.layer_norm_grad(x, x, stats)):
        assert _same_bits(a, v)
    u = torch.rand(3, device="cuda")
    for how in (dict(), dict(top_k=9), dict(top_p=0.9)):
        assert all(_same_bits(a, v) for a, v in zip(B.sample(rows, u, **how), B.sample(x, u, **how)))
    # outputs there
    want = B.embed(torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), x, 3.0)
    assert _same_bits(B.embed(torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda"), x, 3.0, out=rows), want)
    want = B.embed_grad(ids, _normal(3, 5, c, dtype=torch.bfloat16), 3)
    assert _same_bits(B.embed_grad(ids, _normal(3, 5, c, dtype=torch.bfloat16), 3, out=rows), want)
    want = B.dropout(x, 0.5, _seed())
    assert _same_bits(B.dropout(x, 0.5, _seed(), out=rows), want)
    assert _same_bits(B.layer_norm(x, out=rows)[0], B.layer_norm(x)[0])


def test_more_workgroups_than_a_launch_takes():
    """Very long rows: parts of several launches, columns near 2^31."""
    w = 1_500_000_007
    x = torch.ones(3, w, dtype=torch.bfloat16, device="cuda")
    B.dropout(x, 0.5, _seed(), out=x)
    units = (w + 7) // 8
    for r in range(3):
        for first in (0, (2 ** 21 * 256 - r * units) % units, units - 40):
            first = min(first, units - 40)
            unit, row = np.arange(first, first + 40, dtype=np.uint64), np.full(40, r, np.uint64)
            words = L.random_words(unit, row, np.full(40, 7, np.uint64), np.zeros(40, np.uint64),
                                   1234567890123 % 2 ** 32, 1234567890123 >> 32)
            half = np.stack([h for v in words for h in (v & np.uint64(0xFFFF), v >> np.uint64(16))], 1).reshape(-1)
            got = np64(x[r, first * 8:first * 8 + 320])
            assert np.array_equal(got != 0, (half >= 32768)[:len(got)]), (r, first)
    table = x[:2]
    ids = torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
    out = B.embed(ids, table, 2.0)
    for r, e in enumerate((1, 0, 1)):
        for part in (slice(0, 5000), slice(w // 2, w // 2 + 5000), slice(w - 5000, w)):
            assert torch.equal(out[r, part], table[e, part] * 2)
    del out
    y, _ = B.layer_norm(table)
    # zeros and twos in equal shares: -1 and 1 to about 2^-15, half a step of the output
    assert torch.equal(y[1, -5000:], (table[1, -5000:] - 1).sign())
    assert torch.equal(y[0, w // 3:w // 3 + 5000], (table[0, w // 3:w // 3 + 5000] - 1).sign())


def test_sample_more_rows_than_a_launch_takes():
    n = (1 << 20) + 77
    z, u = _normal(1, n, 3), torch.rand(n, device="cuda", generator=_gen(2))
    ids, _ = B.sample(z, u)
    w = torch.cumsum(torch.softmax(z.double(), 1), 1)
    want = (w <= u.double()[:, None]).sum(1).clamp(max=2)
    near = (w - u.double()[:, None]).abs().min(1).values < 1e-12
    assert bool(((ids == want) | near).all())


def test_refused_tensors():
    x, ids, w = _normal(1, 6, 8), torch.zeros(6, 2, dtype=torch.int32, device="cuda"), _normal(2, 8)
    seed, u, stats = _seed(), torch.rand(6, device="cuda"), torch.empty(6, 3, device="cuda")
    half = x.half()
    wrong = [
        (TypeError, lambda: B.embed(ids.long(), x)), (TypeError, lambda: B.embed(ids, x.double())),
        (TypeError, lambda: B.embed(ids, x.int())), (ValueError, lambda: B.embed(ids, x.t())),
        (ValueError, lambda: B.embed(ids.t(), x)), (ValueError, lambda: B.embed(ids, x[0])),
        (ValueError, lambda: B.embed(ids, x, offsets=torch.zeros(2, dtype=torch.int64, device="cuda"))),
        (TypeError, lambda: B.embed(ids, x, offsets=torch.zeros(3, device="cuda"))),
        (ValueError, lambda: B.embed(ids[:1, 0].expand(6), x)),
        (ValueError, lambda: B.embed(ids, x, out=torch.empty(5, 8, device="cuda"))),
        (TypeError, lambda: B.embed(ids, x, out=half)), (B.BridgerError, lambda: B.embed(ids, x, out=x)),
        (B.BridgerError, lambda: B.embed(ids, x, scale=inf)), (B.BridgerError, lambda: B.embed(ids[:, :0], x)),
        (ValueError, lambda: B.embed_grad(ids, x, 0)), (ValueError, lambda: B.embed_grad(ids, x, 2 ** 31)),
        (ValueError, lambda: B.embed_grad(ids, x[:5], 4)), (ValueError, lambda: B.embed_grad(ids, x, 4, out=x)),
        (B.BridgerError, lambda: B.embed_grad(ids, x, 6, out=x)),
        (TypeError, lambda: B.dropout(x, 0.5, seed.int())), (ValueError, lambda: B.dropout(x, 0.5, seed[:1])),
        (TypeError, lambda: B.dropout(x, 0.5, 7)), (B.BridgerError, lambda: B.dropout(x, 1.5, seed)),
        (B.BridgerError, lambda: B.dropout(x, nan, seed)), (ValueError, lambda: B.dropout(x, 0.5, seed, layer=-1)),
        (ValueError, lambda: B.dropout(x, 0.5, seed, layer=2 ** 31)), (TypeError, lambda: B.dropout(x, 0.5, seed, half)),
        (ValueError, lambda: B.dropout(x, 0.5, seed, x[:, :7])), (TypeError, lambda: B.dropout(x.double(), 0.5, seed)),
        (ValueError, lambda: B.dropout(x[:1].expand(6, 8), 0.5, seed)), (ValueError, lambda: B.dropout(x[:, ::2], 0.5, seed)),
        (TypeError, lambda: B.layer_norm(x, w.half())), (ValueError, lambda: B.layer_norm(x, w[:7])),
        (ValueError, lambda: B.layer_norm(x, w, w[:7])), (B.BridgerError, lambda: B.layer_norm(x, eps=-1.0)),
        (ValueError, lambda: B.layer_norm(x, stats=stats[:, :2])), (TypeError, lambda: B.layer_norm(x, stats=stats.half())),
        (B.BridgerError, lambda: B.layer_norm(x, out=x)), (TypeError, lambda: B.layer_norm(x, residual=half)),
        (ValueError, lambda: B.layer_norm_grad(x, x[:5], stats)), (TypeError, lambda: B.layer_norm_grad(x, half, stats)),
        (ValueError, lambda: B.layer_norm_grad(x, x, stats[:5])), (B.BridgerError, lambda: B.layer_norm_grad(x, x, stats, out=x)),
        (TypeError, lambda: B.layer_norm_grad(x, x, stats, grad_total=half)),
        (TypeError, lambda: B.sample(x, u.double())), (ValueError, lambda: B.sample(x, u[:5])),
        (B.BridgerError, lambda: B.sample(x, u, temperature=-1.0)), (ValueError, lambda: B.sample(x, u, top_k=-1)),
        (ValueError, lambda: B.sample(x, u, top_k=2 ** 31)), (B.BridgerError, lambda: B.sample(x, u, top_p=1.5)),
        (B.BridgerError, lambda: B.sample(x, u, min_p=nan)), (TypeError, lambda: B.sample(x, u, top_k=u)),
        (TypeError, lambda: B.sample(x, u, temperature=u.double())), (ValueError, lambda: B.sample(x, u, top_p=u[:3])),
        (TypeError, lambda: B.sample(x.long(), u)), (ValueError, lambda: B.sample(x, u, ids=ids[:, 0])),
        (B.BridgerError, lambda: B.sample(x, u, logp=u)),
    ]
    for i, (error, call) in enumerate(wrong):
        with pytest.raises(error):
            call()
            pytest.fail(f"call {i} was not refused")
    torch.cuda.synchronize()


def test_outputs_that_autograd_tracks_or_saves():
    """What is written counts as written in place; what requires grad is refused."""
    x, u, ids = _normal(1, 6, 8), torch.rand(6, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    stats = torch.empty(6, 3, device="cuda")
    B.layer_norm(x, stats=stats)
    for make in (lambda o: B.embed(ids, x, out=o), lambda o: B.embed_grad(ids, x, 6, out=o),
                 lambda o: B.dropout(x, 0.5, _seed(), out=o), lambda o: B.layer_norm(x, out=o),
                 lambda o: B.layer_norm(x, total=o), lambda o: B.layer_norm_grad(x, x, stats, out=o)):
        out = torch.zeros(6, 8, device="cuda")
        before = out._version
        make(out)
        assert out._version > before
        leaf = torch.zeros(6, 8, device="cuda", requires_grad=True)
        with pytest.raises(RuntimeError, match="requires grad"):
            make(leaf)
        with torch.no_grad():
            make(leaf)
    logp, drawn = torch.zeros(6, device="cuda"), torch.zeros(6, dtype=torch.int32, device="cuda")
    before = logp._version, drawn._version
    B.sample(x, u, ids=drawn, logp=logp)
    assert logp._version > before[0] and drawn._version > before[1]
    with pytest.raises(RuntimeError, match="requires grad"):
        B.sample(x, u, logp=torch.zeros(6, device="cuda", requires_grad=True))
    # an input changed between forward and backward
    leaf = _normal(2, 6, 8).requires_grad_()
    h = leaf * 1
    y, _ = B.layer_norm(h)
    h.mul_(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()
    some = ids.clone()
    y = B.embed(some, leaf)
    some.add_(1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.sum().backward()


def test_negated_views():
    """Rows of one element, the only ones whose negated views look dense, are refused; as gradients they are
    resolved."""
    z = torch.complex(_normal(1, 6, 1), _normal(2, 6, 1))
    neg, seed, u = z.conj().imag, _seed(), torch.rand(6, device="cuda")
    ids, stats = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.empty(6, 3, device="cuda")
    for call in (lambda: B.dropout(neg, 0.5, seed), lambda: B.layer_norm(neg), lambda: B.embed(ids, neg),
                 lambda: B.embed_grad(ids, neg, 3), lambda: B.layer_norm_grad(neg, neg, stats), lambda: B.sample(neg, u)):
        with pytest.raises(ValueError, match="resolve_neg"):
            call()
    for n in (1, 6):
        up, x = z[:n].conj().imag, _normal(3, n, 1).requires_grad_()
        assert up.is_neg()
        plain = up.resolve_neg()
        for f in (lambda: B.dropout(x, 0.0, seed), lambda: B.layer_norm(x, x[0])[0], lambda: B.layer_norm(x, None, x[0])[0],
                  lambda: B.embed(ids[:1].expand(n).contiguous(), x)):
            got, = torch.autograd.grad(f(), x, up)
            want, = torch.autograd.grad(f(), x, plain)
            assert torch.equal(got, want)


@pytest.mark.parametrize("gap", [0, 3])
def test_hooks_on_saved_tensors(gap):
    """Gradients from saved tensors that hooks gave in place of the ones saved, laid out otherwise."""
    def pack(t):
        return t.clone()

    def unpack(t):
        if t.dim() == 2 and t.is_floating_point() and gap and t.shape[1] > 3:
            return _strided(t, gap)[1]
        return t.clone()
    x, res, w, b = (t.requires_grad_() for t in _norm_inputs(1, 12, 20, torch.float32))
    ids, seed, up = _ids(2, 12, 3, [4, 5, 3]), _seed(), _normal(3, 12, 20)
    calls = [(lambda: B.layer_norm(x, w, b, residual=res)[0], (x, res, w, b)), (lambda: B.dropout(x, 0.3, seed, res), (x, res)),
             (lambda: B.embed(ids, x, 0.5), (x,)), (lambda: B.layer_norm(x, w)[0], (x, w))]
    for f, leaves in calls:
        want = torch.autograd.grad(f(), leaves, up)
        with torch.autograd.graph.saved_tensors_hooks(pack, unpack):
            out = f()
        got = torch.autograd.grad(out, leaves, up)
        assert all(_same_bits(a, v) for a, v in zip(got, want))


def test_backward_twice_and_in_another_stream():
    """A graph that is kept gives the same gradients again, in tensors of their own."""
    x, res, w, b = (t.requires_grad_() for t in _norm_inputs(1, 300, 257, torch.bfloat16))
    up = _normal(3, 300, 257, dtype=torch.bfloat16)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y, _ = B.layer_norm(B.dropout(x, 0.2, _seed(), res), w, b)
    first = torch.autograd.grad(y, (x, res, w, b), up, retain_graph=True)
    second = torch.autograd.grad(y, (x, res, w, b), up)
    torch.cuda.synchronize()
    for p, q in zip(first, second):
        assert p.data_ptr() != q.data_ptr() and _same_bits(p, q)
