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
    """Sums in the order of the rows: equal bits whatever else runs, and those of a sum in order
    where an entry has few rows."""
    ids = _ids(3, 5000, 1, [900], empty=0.0)[:, 0]
    grad = _normal(4, 5000, 24)
    first = B.embed_grad(ids, grad, 900)
    for _ in range(5):
        assert _same_bits(first, B.embed_grad(ids, grad, 900))
    want = np.zeros((900, 24), np.float32)
    g, at, count = grad.cpu().numpy(), ids.cpu().numpy(), np.bincount(ids.cpu().numpy(), minlength=900)
    for r in range(5000):
        want[at[r]] += g[r]
    few = count <= 32
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
