"""The row operators on the GPU against their definitions in 64 bits (operators_ref.py): types,
widths from one to long rows, odd sizes and strides, empty and masked rows, NaN and infinities, far
offsets, streams and captured graphs, and a run of them together with a forest."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

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
    kind = {4: torch.int32, 2: torch.int16, 1: torch.int8}[a.element_size()]
    return torch.equal(a.contiguous().view(kind), b.contiguous().view(kind))


WIDTHS = [1, 2, 3, 7, 10, 31, 63, 64, 65, 100, 255, 256, 257, 511, 513, 784, 1000, 1024, 2047, 2049,
          4096, 5001, 8192, 8195, 16384, 33001, 65536, 65543, 131072, 150001]


# ------------------------------------------------------------------------------ top_k
def _check_top(scores, k, values, ids, what=""):
    v, i = R.top_k(scores, k)
    assert np.array_equal(ids.cpu().numpy(), i), f"{what}: ids"
    got = np64(values)
    assert np.array_equal(np.isnan(got), np.isnan(v)) and np.array_equal(got[~np.isnan(v)], v[~np.isnan(v)]), what


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", WIDTHS)
def test_top_k(width, dtype):
    n = 5 if width > 1000 else 37
    s = _normal(width, n, width, scale=3, dtype=dtype)
    for k in sorted({1, 4, min(width, 20), min(width + 3, 64), 256}):
        values, ids = B.top_k(s, k)
        _check_top(s, k, values, ids, f"{width} {dtype} k={k}")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [5, 64, 300, 4096, 20000, 140000])
def test_top_k_ties_and_orders(width, dtype):
    """Equal values, rows in either order, one value standing out, values of one lane's stride."""
    j = torch.arange(width, device="cuda", dtype=torch.float32)
    far = torch.finfo(dtype).max
    rows = [torch.zeros(width, device="cuda"), (j % 3), (j % 1000) / 8, -((j % 777) / 8),
            torch.where(j == width - 1, 1.0, 0.0), torch.where(j == 0, -1.0, 0.0),
            torch.where(j % 1024 == 5, 2.0, -2.0), torch.where(j % 64 == 3, far, -far),
            torch.where(j % 2 == 0, 0.0, -0.0), torch.full((width,), -far, device="cuda"),
            j.clamp(max=60000), 60000 - j.clamp(max=60000), torch.floor(j / 8), -torch.floor(j / 8)]
    s = torch.stack(rows).to(dtype)
    for k in (1, 7, 64, 256):
        values, ids = B.top_k(s, k)
        _check_top(s, k, values, ids, f"k={k}")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [3, 50, 700, 9000, 70000])
def test_top_k_masked_and_broken(width, dtype):
    s = _normal(1, 12, width, dtype=dtype)
    s[0] = -inf
    s[1] = nan
    s[2] = inf
    s[3, ::2] = nan
    s[4, 1:] = -inf
    s[5, :-1] = nan
    s[6, ::3] = -inf
    s[7, -1] = inf
    s[8, 0] = nan
    s[9] = torch.finfo(dtype).min
    s[9, -1] = -inf
    for k in (1, 3, 100):
        values, ids = B.top_k(s, k)
        _check_top(s, k, values, ids, f"k={k}")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width,gap,lead", [(10, 1, 1), (65, 3, 1), (1000, 7, 3), (5000, 1, 0), (70001, 2, 5)])
def test_top_k_strided(width, gap, lead, dtype):
    _, s = _strided(_normal(2, 9, width, dtype=dtype), gap, lead, fill=100.0)
    values, ids = B.top_k(s, 8)
    _check_top(s, 8, values, ids)
    only = torch.full((9, 8), 9, dtype=torch.int32, device="cuda")
    B.bridger_top_k(s.data_ptr(), s.stride(0), {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[dtype],
                    9, width, 8, None, only.data_ptr(), torch.cuda.current_stream().cuda_stream)
    assert torch.equal(only, ids)


@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 4097, 100_003])
def test_top_k_rows(n):
    s = _normal(n, n, 10)
    buf = torch.full((n + 3, 4), 7, dtype=torch.int32, device="cuda")
    values, ids = B.top_k(s, 4, ids=buf[:n])
    _check_top(s, 4, values, ids)
    assert (buf[n:] == 7).all()


def test_top_k_no_rows():
    values, ids = B.top_k(torch.empty(0, 10, device="cuda"), 3)
    assert values.shape == ids.shape == (0, 3)


# ----------------------------------------------------------------------------- distill
def _teacher(seed, n, c, k, dtype=torch.float32, empty=0.1):
    g = _gen(seed)
    ids = torch.stack([torch.randperm(c, generator=g, device="cuda")[:k] if c >= k else
                       torch.randint(0, c, (k,), generator=g, device="cuda") for _ in range(n)]).to(torch.int32)
    ids[torch.rand(n, k, generator=g, device="cuda") < empty] = -1
    t = (torch.randn(n, k, generator=g, device="cuda") * 3).to(dtype)
    return ids, t


def _check_distill(z, ids, t, T, w=None, what="", backward=True):
    ref_loss, ref_grad, loss_tol, grad_tol = R.distill(z, ids, t, T, w)
    loss, grad = B.distill(z, ids, t, T, weight=w)
    R.assert_near(loss, ref_loss, loss_tol, torch.float32, f"{what}: loss")
    R.assert_near(grad, ref_grad, grad_tol, z.dtype, f"{what}: gradient")
    if backward:
        leaf = z.detach().clone().requires_grad_()
        again = B.distill_loss(leaf, ids, t, T)
        R.assert_near(again, ref_loss, loss_tol, torch.float32, f"{what}: loss alone")
        up = w if w is not None else torch.ones_like(loss)
        got, = torch.autograd.grad(again, leaf, up)
        R.assert_near(got, ref_grad, grad_tol, z.dtype, f"{what}: gradient alone")
    return loss, grad


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", WIDTHS)
def test_distill(width, dtype):
    n = 3 if width > 1000 else 21
    k = min(width, 20)
    z = _normal(width, n, width, scale=3, dtype=dtype)
    for seed, (T, kk, tt) in enumerate([(1.0, k, dtype), (2.5, 1, torch.float32), (0.5, min(width, 200), torch.bfloat16)]):
        ids, t = _teacher(seed, n, width, kk, tt, empty=0.1 if kk > 1 else 0.0)
        w = torch.rand(n, device="cuda", generator=_gen(seed)) + 0.1 if seed != 1 else None
        _check_distill(z, ids, t, T, w, f"{width} {dtype} T={T} k={kk}")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [1, 9, 100, 700, 3000, 40000, 140000])
def test_distill_masked_and_empty(width, dtype):
    k = 6
    z = _normal(3, 14, width, scale=2, dtype=dtype)
    ids, t = _teacher(4, 14, width, k, torch.float32, empty=0.0)
    low = torch.finfo(dtype).min
    ids[0] = -1                                   # no slot is filled
    t[1] = -inf                                   # filled with nothing
    ids[2] = width                                # outside the classes
    ids[3, 1:] = width + 5
    t[4, ::2] = -inf
    z[5] = low                                    # nothing but the type's lowest value
    z[6, 1:] = low
    z[7, ::2] = -inf
    z[7, ids[7].long()] = 0.5                     # the masked classes are not wanted
    z[8] = -inf                                   # no class left, some wanted: loss +infinity
    z[9, ids[9, 0].long()] = -inf                 # a wanted class is masked
    ids[10] = ids[10, 0].clone()                  # one class in every slot
    ids[11, 3] = ids[11, 1]
    z[12] = -inf
    ids[12] = -1                                  # nothing on either side
    t[13] = torch.finfo(torch.float32).min
    for T in (1.0, 4.0):
        loss, grad = _check_distill(z, ids, t, T, None, f"{width} T={T}")
        assert loss[8] == inf and loss[9] == inf
        for r in (0, 1, 2, 12):
            assert loss[r] == 0 and (grad[r] == 0).all()


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [10, 600, 9000, 70000])
def test_distill_broken_rows(width, dtype):
    z = _normal(3, 8, width, dtype=dtype)
    ids, t = _teacher(4, 8, width, 4, empty=0.0)
    z[0, width // 2] = nan
    z[1, -1] = inf
    t[2, 1] = nan
    t[3, 0] = inf
    z[4] = nan
    t[5] = nan
    ids[6] = -1
    z[6, 0] = nan                                 # an empty row hides it
    loss, grad = B.distill(z, ids, t, 2.0)
    leaf = z.clone().requires_grad_()
    alone = B.distill_loss(leaf, ids, t, 2.0)
    late, = torch.autograd.grad(alone.sum(), leaf)
    for lo, g in ((loss, grad), (alone, late)):
        assert torch.isnan(lo[[0, 1, 2, 3, 4, 5]]).all()
        assert torch.isnan(g[[0, 1, 4]]).all()
        assert lo[6] == 0 and (g[6] == 0).all()
        for r in (2, 3, 5):
            assert torch.isnan(g[r, ids[r, 0].long()])
    _check_distill(z[7:], ids[7:], t[7:], 2.0)


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width,gap,lead", [(10, 3, 1), (129, 1, 1), (1000, 7, 3), (5000, 1, 1), (70001, 3, 5), (140003, 1, 1)])
def test_distill_strided_and_in_place(width, gap, lead, dtype):
    z0 = _normal(5, 7, width, scale=2, dtype=dtype)
    ids, t = _teacher(6, 7, width, 8)
    zb, z = _strided(z0, gap, lead, fill=5.0)
    gb, g = _strided(torch.zeros_like(z0), gap + 2, lead + 1, fill=7.0)
    _, ref, _, tol = R.distill(z, ids, t, 1.5)
    loss, _ = B.distill(z, ids, t, 1.5, grad=g)
    R.assert_near(g, ref, tol, dtype)
    assert _untouched(gb, g, 7.0) and torch.equal(z, z0)
    # the same bits whatever the alignment, and where the gradient takes the logits' place
    loss0, g0 = B.distill(z0, ids, t, 1.5)
    assert _same_bits(g0, g) and _same_bits(loss, loss0)
    loss1, _ = B.distill(z, ids, t, 1.5, grad=z)
    assert _same_bits(z, g0) and _same_bits(loss1, loss0) and _untouched(zb, z, 5.0)


def test_distill_gradient_against_differences():
    """The gradient that comes out, against differences of the loss in 64 bits."""
    z = _normal(7, 4, 12, scale=1.0)
    ids, t = _teacher(8, 4, 12, 5)
    _, grad = B.distill(z, ids, t, 1.7)
    base = z.double().cpu()
    for j in range(12):
        h = 1e-4
        up, dn = base.clone(), base.clone()
        up[:, j] += h
        dn[:, j] -= h
        d = (R.distill(up, ids, t, 1.7)[0] - R.distill(dn, ids, t, 1.7)[0]) / (2 * h)
        # differences: h^2 / 6 times a third derivative of at most 1 / T, and 1e-15 / h of rounding
        assert np.abs(np64(grad[:, j]) - d).max() < 1e-6


@pytest.mark.parametrize("n", [1, 3, 64, 1025, 30_001])
def test_distill_rows(n):
    z, (ids, t) = _normal(n, n, 10, scale=2), (torch.randint(-1, 10, (n, 4), device="cuda", dtype=torch.int32, generator=_gen(n)),
                                              _normal(n + 1, n, 4))
    _check_distill(z, ids, t, 2.0, torch.rand(n, device="cuda", generator=_gen(2)))


def test_distill_extreme_temperatures():
    z = _normal(9, 6, 50, scale=2)
    ids, t = _teacher(10, 6, 50, 5, empty=0.0)
    for T in (1e-3, 1e3):
        _check_distill(z, ids, t, T, None, f"T={T}")
    for T in (1e-6, 1e6):
        loss, grad = B.distill(z, ids, t, T)
        assert torch.isfinite(loss).all() and torch.isfinite(grad).all()


@pytest.mark.parametrize("width", [3, 40, 700, 30000, 280000])
def test_distill_kept_classes_of_the_lowest_value(width):
    """z / T leaves float for T below 1, the loss does not."""
    z = _normal(1, 4, width)
    ids, t = _teacher(2, 4, width, 2, empty=0.0)
    z[1, ids[1, 0]] = torch.finfo(torch.float32).min
    z[2] = torch.finfo(torch.float32).min
    z[2, ids[2, 1]] = 0
    z[3, ids[3].long()] = torch.finfo(torch.float32).min
    loss, _ = _check_distill(z, ids, t, 0.5, None, f"{width}")
    assert bool(torch.isfinite(loss).all())
    # one class in three slots, whose p add up to a step more than 1
    same = torch.ones(4, 3, dtype=torch.int32, device="cuda")
    three = torch.tensor([-0.35896924138069153, 0.1679827868938446, 4.211813926696777], device="cuda").repeat(4, 1)
    z[1, 1] = torch.finfo(torch.float32).min
    loss, _ = _check_distill(z, same, three, 0.5, None, f"{width}")
    assert bool(torch.isfinite(loss).all())
    ids[:, 0], ids[:, 1], t[:, 0], t[:, 1] = 0, 1, 3.0, -3.0   # p of 0.82 and 0.18 at T = 4
    z[1:, :], z[1, 1] = 0, torch.finfo(torch.float32).min
    loss, _ = _check_distill(z, ids, t, 4.0, None, f"{width}")
    assert bool(torch.isfinite(loss).all()) and float(loss[1]) > 1e38


def test_distill_no_rows():
    z = torch.empty(0, 9, device="cuda", requires_grad=True)
    loss = B.distill_loss(z, torch.empty(0, 2, dtype=torch.int32, device="cuda"), torch.empty(0, 2, device="cuda"))
    g, = torch.autograd.grad(loss.sum(), z)
    assert loss.shape == (0,) and g.shape == (0, 9)


def test_distill_loss_in_autograd():
    """Broadcast upstream gradients, a leaf used twice, logits that are no leaf, no second derivative."""
    z = _normal(11, 6, 33, scale=2)
    ids, t = _teacher(12, 6, 33, 4)
    _, ref, _, tol = R.distill(z, ids, t, 2.0)
    leaf = z.clone().requires_grad_()
    B.distill_loss(leaf, ids, t, 2.0).mean().backward()
    R.assert_near(leaf.grad, ref / 6, tol / 6 + np.abs(ref) * R.U, torch.float32)
    leaf = z.clone().requires_grad_()
    (B.distill_loss(leaf, ids, t, 2.0).sum() + B.distill_loss(leaf, ids, t, 2.0).sum()).backward()
    R.assert_near(leaf.grad, 2 * ref, 2 * tol + 2 * np.abs(ref) * R.U, torch.float32)
    leaf = z.clone().requires_grad_()
    B.distill_loss(leaf * 1.0, ids, t, 2.0).sum().backward()
    R.assert_near(leaf.grad, ref, tol, torch.float32)
    g, = torch.autograd.grad(B.distill_loss(leaf, ids, t, 2.0).sum(), leaf, create_graph=True)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(g.sum(), leaf)


@pytest.mark.parametrize("gap", [0, 5])
def test_distill_loss_with_hooks_on_saved_tensors(gap):
    """Saved tensors that come back from the host, where they lose the distance between rows."""
    base = _normal(1, 40, 300 + gap, dtype=torch.bfloat16).requires_grad_()
    ids, t = _teacher(2, 40, 300, 5)
    up = torch.rand(40, device="cuda")
    plain, = torch.autograd.grad(B.distill_loss(base[:, :300], ids, t, 2.0), base, up)
    with torch.autograd.graph.save_on_cpu():
        loss = B.distill_loss(base[:, :300], ids, t, 2.0)
    again, = torch.autograd.grad(loss, base, up)
    assert _same_bits(plain, again)


def test_distill_loss_is_differentiated_once():
    z = _normal(1, 6, 50).requires_grad_()
    ids, t = _teacher(2, 6, 50, 5)
    grad, = torch.autograd.grad(B.distill_loss(z, ids, t).sum(), z, create_graph=True)
    plain, = torch.autograd.grad(B.distill_loss(z, ids, t).sum(), z)
    assert _same_bits(grad.detach(), plain)
    with pytest.raises(RuntimeError):
        torch.autograd.grad(grad.square().sum(), z)
    loss = B.distill_loss(z, ids, t)
    ids.add_(1)                            # what the backward pass needs has changed
    with pytest.raises(RuntimeError):
        loss.sum().backward()


# -------------------------------------------------------------------------- rmsnorm_q8
def _check_norm(x, w, r, eps=1e-6, what="", **out):
    before = [None if v is None else v.clone() for v in (x, r)]
    q, scale, total = B.rmsnorm_q8(x, w, r, eps, **out)
    R.check_rmsnorm(before[0], w, before[1], eps, q, scale, total, what)
    return q, scale, total


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", WIDTHS)
def test_rmsnorm(width, dtype):
    n = 4 if width > 1000 else 37
    x, r = _normal(width, n, width, scale=2, dtype=dtype), _normal(width + 1, n, width, dtype=dtype)
    w = _normal(width + 2, width, dtype=dtype)
    _check_norm(x, w, r, what=f"{width} {dtype}")
    _check_norm(x, w, None, what=f"{width} {dtype} no residual")
    _check_norm(x, None, r, 0.5, what=f"{width} {dtype} no weight")
    total = torch.empty_like(x)
    _check_norm(x, None, None, 0.0, what=f"{width} {dtype} bare", total=total)
    assert _same_bits(total, x)


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [1, 12, 64, 300, 1500, 9000, 40001])
def test_rmsnorm_zeros_and_broken(width, dtype):
    x = _normal(1, 12, width, dtype=dtype)
    big, small = torch.finfo(dtype).max, torch.finfo(dtype).tiny
    x[0] = 0
    x[1, -1] = nan
    x[2, 0] = inf
    x[3] = -inf
    x[4] = big
    x[5] = small
    x[6] = 0
    x[6, width // 2] = 1
    x[7] = -0.0
    x[8, 0] = big
    x[9] = small * torch.finfo(dtype).eps
    w = _normal(2, width, dtype=dtype) + 2
    for eps in (1e-6, 0.0):
        for weight in (w, None):
            _check_norm(x, weight, None, eps, f"eps={eps}")
        _check_norm(x, w, x.clone(), eps, f"eps={eps}, residual")      # big + big passes float
        _check_norm(x, w * 0, None, eps, "weights of zero")
    w[-1] = nan
    _check_norm(x, w, None, what="a NaN weight")
    tiny = torch.full_like(w, small)
    tiny[-1] = small * 4
    _check_norm(x, tiny, None, what="tiny weights")
    _check_norm(x, torch.full_like(w, big / 4), None, what="huge weights")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width,gap,lead", [(10, 3, 1), (65, 1, 1), (784, 5, 3), (4096, 1, 1), (9001, 3, 5), (40001, 1, 1)])
def test_rmsnorm_strided_and_in_place(width, gap, lead, dtype):
    x0, r0 = _normal(1, 7, width, dtype=dtype), _normal(2, 7, width, dtype=dtype)
    w = _normal(3, width + lead, dtype=dtype)[lead:]
    xb, x = _strided(x0, gap, lead, 3.0)
    rb, r = _strided(r0, gap + 1, lead + 2, 3.0)
    qb, q = _strided(torch.zeros(7, width, dtype=torch.int8, device="cuda"), gap, lead, 77)
    tb, t = _strided(torch.zeros_like(x0), gap + 2, lead + 1, 9.0)
    _, scale, _ = _check_norm(x, w, r, q=q, total=t)
    assert _untouched(qb, q, 77) and _untouched(tb, t, 9.0)
    assert torch.equal(x, x0) and torch.equal(r, r0)
    q0, scale0, t0 = B.rmsnorm_q8(x0, w, r0)
    assert torch.equal(q0, q) and _same_bits(scale, scale0) and _same_bits(t, t0)
    q1, scale1, _ = B.rmsnorm_q8(x, w, r, total=x)               # the sum in x's place
    assert torch.equal(q1, q0) and _same_bits(scale1, scale0) and _same_bits(x, t0)
    assert _untouched(xb, x, 3.0)
    x.copy_(x0)
    q1, scale1, _ = B.rmsnorm_q8(x, w, r, total=r)               # in the residual's
    assert torch.equal(q1, q0) and _same_bits(scale1, scale0) and _same_bits(r, t0) and torch.equal(x, x0)
    assert _untouched(rb, r, 3.0)
    q2, scale2, t2 = B.rmsnorm_q8(x0, w, x0)                     # one tensor twice
    R.check_rmsnorm(x0, w, x0, 1e-6, q2, scale2, t2)


@pytest.mark.parametrize("n", [1, 2, 63, 65, 1025, 40_003])
def test_rmsnorm_rows(n):
    _check_norm(_normal(n, n, 28), _normal(1, 28), None)


def test_rmsnorm_no_rows():
    q, scale, total = B.rmsnorm_q8(torch.empty(0, 5, device="cuda"))
    assert q.shape == (0, 5) and scale.shape == (0,) and total is None


# --------------------------------------------------------------------------- matmul_q8
def _int8(seed, n, w):
    return torch.randint(-128, 128, (n, w), generator=_gen(seed), device="cuda", dtype=torch.int8)


def _check_product(n, m, f, dtype, bias=True, seed=0):
    a, b = _int8(seed, n, f), _int8(seed + 1, m, f)
    sa, sb = torch.rand(n, generator=_gen(seed + 2), device="cuda"), torch.rand(m, generator=_gen(seed + 3), device="cuda")
    sa *= 1e-3                               # sums of 131071 features stay within float16
    v = _normal(seed + 4, m) if bias else None
    out = B.matmul_q8(a, sa, b, sb, v, dtype)
    R.check_matmul(a, sa, b, sb, v, out, f"{n} x {f} x {m} {dtype}")


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("n", [1, 2, 7, 16, 17, 31, 33, 64, 65, 100, 128, 129, 200, 257, 513])
@pytest.mark.parametrize("m,f", [(1, 1), (10, 28), (16, 64), (33, 65), (64, 784), (100, 1000), (257, 129), (512, 1024), (1000, 2047), (4099, 96)])
def test_matmul(n, m, f, dtype):
    _check_product(n, m, f, dtype, bias=(n + m) % 2 == 0, seed=n)


@pytest.mark.parametrize("n,m,f", [(1, 3, 131071), (5, 17, 131056), (130, 70, 20000), (300, 5, 9001), (1, 40000, 64),
                                   (2048, 2048, 512), (2049, 1031, 527), (5000, 10, 784), (4096, 4096, 4096), (777, 5000, 1024)])
def test_matmul_large(n, m, f):
    _check_product(n, m, f, torch.float32, seed=n)
    _check_product(n, m, f, torch.bfloat16, bias=False, seed=n)


@pytest.mark.parametrize("n", [1, 20, 200, 600])
def test_matmul_full_range(n):
    """Every factor -128: the largest sums that 32 bits take."""
    f = 131071 if n < 100 else 20000
    a = torch.full((n, f), -128, dtype=torch.int8, device="cuda")
    b = torch.full((40, f), -128, dtype=torch.int8, device="cuda")
    one = torch.ones(max(n, 40), device="cuda")
    out = B.matmul_q8(a, one[:n], b, one[:40], dtype=torch.float32)
    assert (out == float(np.float32(f * 16384))).all()
    b.fill_(127)
    out = B.matmul_q8(a, one[:n], b, one[:40], dtype=torch.float32)
    assert (out == float(np.float32(-f * 128 * 127))).all()


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("n,m,f,gap,lead", [(1, 50, 100, 1, 1), (5, 33, 64, 3, 1), (40, 70, 200, 16, 16), (130, 300, 256, 5, 7),
                                            (300, 257, 512, 16, 0), (600, 520, 1000, 1, 3)])
def test_matmul_strided(n, m, f, gap, lead, dtype):
    a0, b0 = _int8(1, n, f), _int8(2, m, f)
    sa, sb = torch.rand(n, device="cuda", generator=_gen(3)), torch.rand(m, device="cuda", generator=_gen(4)) * 1e-3
    _, a = _strided(a0, gap, lead, 99)
    _, b = _strided(b0, gap + 1, lead + 1, 99)
    ob, o = _strided(torch.zeros(n, m, dtype=dtype, device="cuda"), gap, lead, 11.0)
    out = B.matmul_q8(a, sa, b, sb, out=o)
    assert out is o and _untouched(ob, o, 11.0)
    R.check_matmul(a0, sa, b0, sb, None, o)
    assert _same_bits(o.contiguous(), B.matmul_q8(a0, sa, b0, sb, dtype=dtype))


def test_matmul_scales_of_zero_infinity_and_nan():
    for n in (1, 40, 300):
        a, b = _int8(1, n, 96), _int8(2, 50, 96)
        sa, sb = torch.rand(n, device="cuda"), torch.rand(50, device="cuda")
        sa[0], sb[1], sb[2] = nan, 0.0, nan
        if n > 2:
            sa[1], sa[2] = 0.0, inf
        out = B.matmul_q8(a, sa, b, sb, dtype=torch.float32)
        acc = torch.from_numpy(a.cpu().numpy().astype(np.float64) @ b.cpu().numpy().astype(np.float64).T).float().cuda()
        ref = acc * sa[:, None] * sb[None, :]
        assert torch.equal(torch.isnan(out), torch.isnan(ref))
        assert torch.equal(torch.isinf(out), torch.isinf(ref))


def test_matmul_no_rows():
    out = B.matmul_q8(torch.empty(0, 8, dtype=torch.int8, device="cuda"), torch.empty(0, device="cuda"),
                      _int8(1, 3, 8), torch.ones(3, device="cuda"))
    assert out.shape == (0, 3)


# ------------------------------------------------------------------------ all of them
def _every(seed=0, n=65, c=1030):
    """(name, inputs, call): each operator with its inputs, and what it returns."""
    z, s = _normal(seed, n, c, scale=2, dtype=torch.bfloat16), _normal(seed + 1, n, c)
    ids, t = _teacher(seed + 2, n, c, 8)
    x, r = _normal(seed + 3, n, c, dtype=torch.float16), _normal(seed + 4, n, c, dtype=torch.float16)
    w = _normal(seed + 5, c, dtype=torch.float16)
    a, b = _int8(seed + 6, n, c), _int8(seed + 7, 130, c)
    sa, sb = torch.rand(n, device="cuda"), torch.rand(130, device="cuda")
    stats = torch.empty(n, 2, device="cuda")
    return {
        "top_k": ([s], lambda: B.top_k(s, 9)),
        "distill": ([z, t], lambda: B.distill(z, ids, t, 2.0)),
        "rmsnorm_q8": ([x, r], lambda: B.rmsnorm_q8(x, w, r)),
        "matmul_q8": ([sa, sb], lambda: (B.matmul_q8(a, sa, b, sb),)),
    }, stats


NAMES_ALL = ["top_k", "distill", "rmsnorm_q8", "matmul_q8"]


@pytest.mark.parametrize("name", NAMES_ALL)
@pytest.mark.parametrize("n", [1, 65, 700])
def test_equal_bits_again(name, n):
    call = _every(n=n)[0][name][1]
    first = [v.clone() for v in call() if v is not None]
    for _ in range(5):
        assert all(_same_bits(x, y) for x, y in zip(first, [v for v in call() if v is not None]))


@pytest.mark.parametrize("name", NAMES_ALL)
def test_in_a_graph(name):
    """Captured once, replayed with other inputs in place and eager work between the replays."""
    inputs, call = _every(n=130)[0][name]
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


def test_two_graphs_and_two_streams_side_by_side():
    """Nothing is shared between calls: graphs and streams that run at once give what each gives alone."""
    ops = [_every(seed=k, n=400)[0] for k in (0, 50)]
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
    """Threads with a stream each; one of them is refused again and again, with its own message."""
    from concurrent.futures import ThreadPoolExecutor
    ops = [_every(seed=k, n=300, c=2000)[0] for k in (0, 50, 100)]
    alone = [{k: [v.clone() for v in o[k][1]()] for k in NAMES_ALL} for o in ops]
    torch.cuda.synchronize()

    def work(i):
        with torch.cuda.stream(torch.cuda.Stream()):
            for _ in range(20):
                outs = {k: ops[i][k][1]() for k in NAMES_ALL}
            torch.cuda.current_stream().synchronize()
        return all(_same_bits(x, y) for k in NAMES_ALL for x, y in zip(alone[i][k], outs[k]))

    def refused(_):
        z = ops[0]["distill"][0][0]
        ids, t = _teacher(1, z.shape[0], z.shape[1], 2)
        for _ in range(200):
            with pytest.raises(B.BridgerError, match="temperature"):
                B.distill(z, ids, t, 0.0)
        return True

    with ThreadPoolExecutor(4) as pool:
        assert all([*pool.map(work, range(3)), *pool.map(refused, range(1))])


def test_backward_in_a_graph_beside_an_eager_one():
    """distill gives the gradient without autograd, so a training step is captured while an eager
    graph of the same logits is alive."""
    z = _normal(1, 40, 500, scale=2).requires_grad_()
    ids, t = _teacher(2, 40, 500, 8)
    eager = B.distill_loss(z, ids, t, 2.0).sum()          # alive until its backward below
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.distill(z, ids, t, 2.0)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        loss, grad = B.distill(z, ids, t, 2.0)
    for _ in range(3):
        grad.zero_()
        g.replay()
        torch.cuda.synchronize()
        _, ref, _, tol = R.distill(z, ids, t, 2.0)
        R.assert_near(grad, ref, tol, torch.float32)
    eager.backward()
    R.assert_near(z.grad, ref, tol, torch.float32)


def test_loss_with_a_gradient_is_refused_in_a_graph():
    x = _normal(1, 6, 8).requires_grad_()
    ids, t = _teacher(2, 6, 8, 3)
    eager = B.distill_loss(x, ids, t)
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        with pytest.raises(RuntimeError):
            B.distill_loss(x, ids, t)
        with torch.no_grad():
            loss = B.distill_loss(x, ids, t)
    for _ in range(3):
        loss.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(loss, eager.detach())
    eager.sum().backward()
    assert bool(torch.isfinite(x.grad).all())


def test_far_offsets():
    """Rows whose offsets pass 2^31 elements (and 2^32 bytes)."""
    far = (1 << 31) + 24
    c = 1000
    buf = torch.empty(2 * far + c, dtype=torch.bfloat16, device="cuda")
    rows = torch.as_strided(buf, (3, c), (far, 1))
    z0 = _normal(1, 3, c, scale=2, dtype=torch.bfloat16)
    rows.copy_(z0)
    ids, t = _teacher(2, 3, c, 5)
    values, top = B.top_k(rows, 10)
    _check_top(z0, 10, values, top)
    _check_distill(rows, ids, t, 2.0)
    _check_norm(rows, None, rows.clone().contiguous())
    loss, _ = B.distill(rows, ids, t, 2.0, grad=rows)
    ref_loss, ref, loss_tol, tol = R.distill(z0, ids, t, 2.0)
    R.assert_near(rows, ref, tol, torch.bfloat16)
    out = B.matmul_q8(_int8(3, 3, 64), torch.ones(3, device="cuda"), _int8(4, c, 64), torch.ones(c, device="cuda") * 1e-3, out=rows)
    R.check_matmul(_int8(3, 3, 64), torch.ones(3, device="cuda"), _int8(4, c, 64), torch.ones(c, device="cuda") * 1e-3, None, out)
    del buf, rows, out
    torch.cuda.empty_cache()
    wide = torch.as_strided(torch.empty(2 * far + 256, dtype=torch.int8, device="cuda"), (3, 256), (far, 1))
    wide.copy_(_int8(5, 3, 256))
    one = torch.ones(3, device="cuda")
    R.check_matmul(wide, one, wide, one, None, B.matmul_q8(wide, one, wide, one, dtype=torch.float32))
    many = torch.empty(((1 << 32) + 640) // 64, 64, dtype=torch.int8, device="cuda")     # rows of 2^32 bytes in all
    many[-300:] = _int8(6, 300, 64)
    sm = torch.ones(many.shape[0], device="cuda")
    out = B.matmul_q8(many, sm, _int8(7, 16, 64), torch.ones(16, device="cuda"), dtype=torch.bfloat16)
    R.check_matmul(many[-300:], sm[-300:], _int8(7, 16, 64), torch.ones(16, device="cuda"), None, out[-300:])
    q, scale, _ = B.rmsnorm_q8(out, None)
    R.check_rmsnorm(out[-300:], None, None, 1e-6, q[-300:], scale[-300:], None)
    values, top = B.top_k(out, 3)
    _check_top(out[-300:], 3, values[-300:], top[-300:])


def test_refused_tensors():
    x = _normal(1, 6, 8)
    ids, t = _teacher(2, 6, 8, 3)
    q, v = _int8(1, 6, 8), torch.ones(6, device="cuda")
    bad = [
        lambda: B.top_k(x.t(), 2), lambda: B.top_k(x[0], 2), lambda: B.top_k(x.expand(6, 8)[:1].expand(6, 8), 2),
        lambda: B.top_k(x, 2, values=torch.empty(6, 3, device="cuda")),
        lambda: B.distill(x, ids[:5], t), lambda: B.distill(x, ids, t[:, :2]),
        lambda: B.distill(x, ids, t, weight=v[:5]), lambda: B.distill(x, ids.t().contiguous().t(), t),
        lambda: B.distill(x, ids, t, grad=torch.empty(6, 7, device="cuda")),
        lambda: B.rmsnorm_q8(x, v), lambda: B.rmsnorm_q8(x, None, x[:5]),
        lambda: B.rmsnorm_q8(x, q=q[:, :7]), lambda: B.matmul_q8(q, v, q[:, :7], v),
        lambda: B.matmul_q8(q, v[:5], q, v), lambda: B.matmul_q8(q, v, q, v, bias=v[:3]),
        lambda: B.matmul_q8(q, v, q, v, out=torch.empty(6, 5, device="cuda")),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
    wrong = [lambda: B.top_k(x.double(), 2), lambda: B.top_k(q, 2), lambda: B.distill(x, ids.long(), t),
             lambda: B.distill(x, ids, t, weight=v.double()), lambda: B.rmsnorm_q8(x, x[0].bfloat16()),
             lambda: B.rmsnorm_q8(x, None, x.bfloat16()), lambda: B.matmul_q8(x, v, q, v),
             lambda: B.matmul_q8(q, v.half(), q, v), lambda: B.matmul_q8(q, v, q, v, dtype=torch.float64)]
    for call in wrong:
        with pytest.raises(TypeError):
            call()
    for call in (lambda: B.top_k(x, 0), lambda: B.top_k(x, 257), lambda: B.distill(x, ids, t, 0.0),
                 lambda: B.distill(x, ids, t, nan), lambda: B.rmsnorm_q8(x, eps=-1.0),
                 lambda: B.top_k(torch.empty(4, 0, device="cuda"), 1),
                 lambda: B.rmsnorm_q8(x[:5], total=x.view(-1)[4:44].view(5, 8))):
        with pytest.raises((B.BridgerError, ValueError)):
            call()


def test_refused_counts_past_32_bits():
    """A count that would lose its upper bits on the way: 2^32 + 3 classes are not 3 classes."""
    wide = torch.empty(1, 2**32 + 3, dtype=torch.bfloat16, device="cuda")
    ids, t = _teacher(1, 1, 3, 2)
    one = torch.ones(1, device="cuda")
    q = torch.zeros(1, 1, dtype=torch.int8, device="cuda")
    many = wide.view(torch.int8).view(-1, 1)
    for call in (lambda: B.top_k(wide, 2), lambda: B.distill(wide, ids, t),
                 lambda: B.distill_loss(wide, ids, t), lambda: B.rmsnorm_q8(wide),
                 lambda: B.matmul_q8(q, one, many, one), lambda: B.matmul_q8(many, one, q, one),
                 lambda: B.matmul_q8(many.view(1, -1), one, many.view(1, -1), one),
                 lambda: B.top_k(wide[:, :8], 2**32 + 2), lambda: B.top_k(wide[:, :8], -1)):
        with pytest.raises(ValueError):
            call()


def test_together_with_a_forest():
    """A forest of ten classes teaches a student that answers in 8 bits: its largest scores, the
    student's norm and product, the loss and the gradient; then the student's own labels."""
    from synth import make_workload
    w = make_workload("mc_gbdt_d8", 300)
    w.forest.transform = B.BRIDGER_XFORM_IDENTITY                 # class scores, not probabilities
    X = torch.from_numpy(w.X()).cuda()
    with B.Forest(w.forest) as f:
        scores = f.predict(X)
        teacher, ids = f.predict_top(X, 4)
        labels = f.predict_labels(X)
    _check_top(scores, 4, teacher, ids)
    # class sums are compared in double for the label, as floats for the order
    sure = teacher[:, 0] > teacher[:, 1]
    assert torch.equal(ids[sure, 0], labels[sure])
    gamma, head = 1 + 0.1 * _normal(1, X.shape[1]), _normal(2, 10, X.shape[1])
    q, scale, _ = B.rmsnorm_q8(X, gamma)
    R.check_rmsnorm(X, gamma, None, 1e-6, q, scale, None)
    hs = head.abs().amax(1) / 127
    hq = torch.round(head / hs[:, None]).to(torch.int8)
    z = B.matmul_q8(q, scale, hq, hs, dtype=torch.float32)
    R.check_matmul(q, scale, hq, hs, None, z)
    share = torch.full((X.shape[0],), 1.0 / X.shape[0], device="cuda")
    _check_distill(z, ids, teacher, 2.0, share)
    _check_top(z, 1, *B.top_k(z, 1))


def test_on_another_stream_and_device_context():
    ops, _ = _every(n=33)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    for name in NAMES_ALL:
        here = [v.clone() for v in ops[name][1]()]
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            there = ops[name][1]()
        s.synchronize()
        assert all(_same_bits(x, y) for x, y in zip(here, there)), name


def test_numbers_of_slots():
    """1 to BRIDGER_MAX_TOP slots, more slots than classes, one class in all of them."""
    for c, k in ((7, 256), (300, 255), (5000, 256), (2, 1), (40000, 129)):
        z = _normal(c, 5, c, scale=2)
        ids = torch.randint(-1, c, (5, k), generator=_gen(k), device="cuda", dtype=torch.int32)
        _check_distill(z, ids, _normal(k, 5, k), 1.5, None, f"c={c} k={k}")
    assert math.isfinite(float(B.distill(z, torch.zeros_like(ids), _normal(1, 5, 129))[0].sum()))


@pytest.mark.parametrize("c,k", [(3, 4), (9, 16), (15, 17), (50, 33), (60, 64), (127, 65), (200, 100),
                                 (255, 128), (255, 129), (350, 128), (400, 129), (1100, 70)])
@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
def test_lanes_and_slots(c, k, dtype):
    """Slots in each of a lane's places; one row of several in a wave holds a class twice."""
    n = 70
    z = _normal(c, n, c, scale=2, dtype=dtype)
    ids, t = _teacher(k, n, c, min(c, k), empty=0.0)
    ids, t = (torch.nn.functional.pad(x, (0, k - x.shape[1]), value=-1) for x in (ids, t))
    ids[5, -1] = ids[5, 0]
    ids[66, : k // 2 + 1] = ids[66, 0]
    _check_distill(z, ids, t, 1.5, None, f"c={c} k={k}")


def test_more_rows_than_a_launch_takes():
    """Rows, and tiles, beyond what one dispatch counts go out as several launches."""
    n = (1 << 20) + 1234
    s = _normal(1, n, 70, dtype=torch.bfloat16)
    values, ids = B.top_k(s, 3)                                    # a workgroup a row
    for part in (slice(0, 300), slice((1 << 20) - 150, (1 << 20) + 150), slice(n - 300, n)):
        _check_top(s[part], 3, values[part], ids[part])
    rows, outputs = (1 << 20) + 70, 1100                           # 2^22.5 tiles of 16 x 16
    a, b = _int8(2, rows, 33), _int8(3, outputs, 33)
    sa, sb = torch.rand(rows, device="cuda", generator=_gen(4)), torch.rand(outputs, device="cuda", generator=_gen(5))
    v = _normal(6, outputs)
    out = B.matmul_q8(a, sa, b, sb, v, torch.float32)
    cut = (1 << 30) // 1280 // 256 * 256                           # where the second launch starts
    for part in (slice(0, 100), slice(cut - 100, cut + 100), slice(rows - 100, rows)):
        R.check_matmul(a[part], sa[part], b, sb, v, out[part])
    del a, out
    outputs = (1 << 20) + 33
    a, b = _int8(7, 20, 40), _int8(8, outputs, 40)
    sa, sb = torch.rand(20, device="cuda", generator=_gen(9)), torch.rand(outputs, device="cuda", generator=_gen(10))
    v = _normal(11, outputs)
    R.check_matmul(a, sa, b, sb, v, B.matmul_q8(a, sa, b, sb, v, torch.float32))


@pytest.mark.parametrize("n,m,f", [(600, 600, 256), (64, 512, 4096), (4096, 4100, 200)])
def test_products_in_a_graph(n, m, f):
    """Kernels of more than 64 KB of LDS, captured and replayed."""
    a, b = _int8(1, n, f), _int8(2, m, f)
    sa, sb = torch.rand(n, device="cuda", generator=_gen(3)), torch.rand(m, device="cuda", generator=_gen(4)) * 1e-3
    out = torch.empty(n, m, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        B.matmul_q8(a, sa, b, sb, out=out)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.matmul_q8(a, sa, b, sb, out=out)
    for rep in range(3):
        a.copy_(_int8(10 + rep, n, f))
        sa.mul_(0.5)
        torch.cuda.synchronize()
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        R.check_matmul(a, sa, b, sb, None, out, f"replay {rep}")


def test_autograd_sees_what_the_library_writes():
    """Memory that a backward pass still needs, overwritten by each output that a caller can give."""
    z0 = _normal(1, 6, 50, scale=2)
    ids, t = _teacher(2, 6, 50, 5)
    x, r = _normal(3, 6, 50), _normal(4, 6, 50)
    a, b = _int8(5, 6, 50), _int8(6, 50, 50)
    one, many = torch.ones(6, device="cuda"), torch.ones(50, device="cuda")

    def saved(shape, write, dtype=torch.float32):
        # exp keeps its result for its gradient; whole numbers are kept by index_select
        if dtype.is_floating_point:
            out = _normal(7, *shape).requires_grad_().exp()
            write(out.detach())
        else:
            index = torch.zeros(shape[0] * shape[1], dtype=dtype, device="cuda")
            out = _normal(7, 50).requires_grad_().index_select(0, index)
            write(index.view(shape))
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.sum().backward()

    saved((6, 5), lambda o: B.top_k(z0, 5, values=o))
    saved((6, 5), lambda o: B.top_k(z0, 5, ids=o), torch.int32)
    saved((6, 50), lambda o: B.distill(z0, ids, t, grad=o))
    saved((1, 6), lambda o: B.distill(z0, ids, t, loss=o[0]))
    saved((6, 50), lambda o: B.distill(o, ids, t, grad=o))
    saved((6, 50), lambda o: B.rmsnorm_q8(x, None, r, total=o))
    saved((6, 50), lambda o: B.rmsnorm_q8(o, None, r, total=o))
    saved((6, 50), lambda o: B.rmsnorm_q8(x, None, o, total=o))
    saved((1, 6), lambda o: B.rmsnorm_q8(x, scale=o[0]))
    saved((6, 50), lambda o: B.matmul_q8(a, one, b, many, out=o))
    q = torch.zeros(6, 50, dtype=torch.int8, device="cuda")
    before = q._version
    B.rmsnorm_q8(x, q=q)
    assert q._version > before
    # the logits, and the ids, that distill_loss keeps itself
    for write in (lambda z, i: B.distill(z.detach(), i, t, grad=z.detach()),
                  lambda z, i: B.top_k(z.detach(), 5, ids=i)):
        z, i = (z0 * 1.0).requires_grad_(), ids.clone()
        loss = B.distill_loss(z, i, t)
        write(z, i)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.sum().backward()
    # an output of the call's own tells nobody
    z = (z0 * 1.0).requires_grad_()
    loss = B.distill_loss(z, ids, t)
    B.distill(z, ids, t)
    B.top_k(z, 5)
    loss.sum().backward()


def test_outputs_that_require_grad():
    z = _normal(1, 6, 50).requires_grad_()
    ids, t = _teacher(2, 6, 50, 5)
    a, one = _int8(5, 6, 50), torch.ones(6, device="cuda")
    small = _normal(3, 6, 5).requires_grad_()
    row = _normal(4, 6).requires_grad_()
    before = z.detach().clone()
    calls = [lambda: B.top_k(z, 5, values=small), lambda: B.distill(z, ids, t, grad=z),
             lambda: B.distill(z, ids, t, loss=row), lambda: B.rmsnorm_q8(z, total=z),
             lambda: B.rmsnorm_q8(z, scale=row), lambda: B.rmsnorm_q8(z, None, z * 1.0, total=z),
             lambda: B.matmul_q8(a, one, a, one, out=(_normal(5, 6, 6).requires_grad_() * 1.0))]
    for call in calls:
        with pytest.raises(RuntimeError, match="requires grad"):
            call()
    assert torch.equal(z, before)
    ref = B.distill(before, ids, t)
    with torch.no_grad():                      # as torch's own in-place operations
        version = z._version
        loss, grad = B.distill(z, ids, t, grad=z)
    assert grad is z and z._version > version
    assert _same_bits(loss, ref[0]) and _same_bits(z.detach(), ref[1])


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [2, 3, 10, 600, 9000, 70000, 140000])
def test_distill_masked_kept_class_in_a_broken_row(width, dtype):
    """A row whose only wanted class is masked has loss +infinity, unless its logits hold a NaN or
    +infinity: then there is no distribution, and the loss is NaN as its gradient is."""
    z = _normal(3, 6, width, dtype=dtype)
    at = width // 2
    ids = torch.full((6, 2), -1, dtype=torch.int32, device="cuda")
    ids[:, 0] = at
    t = torch.zeros(6, 2, device="cuda")
    z[:, at] = -inf
    z[1, 0] = nan
    z[2, 0] = inf
    z[3] = nan                                    # everything else is broken
    z[3, at] = -inf
    z[4, 0] = nan
    ids[4, 1], t[4, 1] = 0, -inf                  # kept, but not wanted
    z[5] = -inf
    leaf = z.clone().requires_grad_()
    alone = B.distill_loss(leaf, ids, t, 2.0)
    late, = torch.autograd.grad(alone.sum(), leaf)
    loss, grad = B.distill(z, ids, t, 2.0)
    for lo, g in ((loss, grad), (alone, late)):
        assert lo[0] == inf and lo[5] == inf
        assert torch.isnan(lo[1:5]).all() and torch.isnan(g[1:5]).all()
        # T (q - p), from what is left
        assert torch.isfinite(g[[0, 5]]).all() and (g[[0, 5], at] == -2).all()


def _check_long_row(z, T, most, S, at, what):
    """One row of float or bfloat16 logits whose sum of exponentials, relative to the largest, is S;
    the teacher wants class `at` alone, one of the largest: loss = T^2 log S, and the gradient of
    the other classes is T e^x / S.

    In half steps U of a float, S is off by: the exponents, whose difference, factor and product are
    rounded (3 |x|, with |x| below 2.8 or weighed by e^x), and 2 for the exponential, 12; 32 terms
    added in float, 31; changes of scale by e^2.77 and more, each 12 and 1/16 of the one before, 13;
    the last one, 12; the double sum's rounding, 1; two joins of lanes whose largest are close, of a
    product and an exponential, 4 each, and 10 additions.  Together below 100.  The logarithm is off
    by 4 of its own size with its constant, the products with T and T^2 by 3."""
    n, U = z.shape[1], R.U
    ids = torch.tensor([[at]], dtype=torch.int32, device="cuda")
    t = torch.zeros(1, 1, device="cuda")
    want = T * T * math.log(S)
    tol = T * T * 100 * U + 7 * U * want
    loss, grad = B.distill(z, ids, t, T)
    leaf = z.detach().requires_grad_()
    alone = B.distill_loss(leaf, ids, t, T)
    late, = torch.autograd.grad(alone, leaf)
    for name, lo, g in (("together", loss, grad), ("later", alone, late)):
        off = abs(lo.item() - want)
        assert off <= tol, f"{what} {name}: loss off by {off:.2e} of {tol:.2e}"
        # S, its reciprocal (3), the exponential (2 and three times its exponent) and three products,
        # then the type's rounding.  An exponential below the smallest normal float, 2^-126, is 0:
        # that is T 2^-126 / S of the gradient at most (T = 0.25, 2^24 rising logits, S = 1.4e5:
        # 2.1e-44, 15 of the smallest steps of a float; exponents down to -120, e^-87.3 = 2^-126)
        worst = 0.0
        for part in torch.arange(n, device="cuda").split(1 << 23):
            x = (z[0, part].double() - most) / T
            ref = T * torch.exp(x) / S
            err = (g[0, part].double() - ref).abs()
            most_off = ref * ((108 + 3 * x.abs()) * U * (1 + R.HALF[z.dtype]) + R.HALF[z.dtype])
            most_off += R.TINY[z.dtype] + T * 2.0 ** -126 / S
            err[part == at] = 0
            worst = max(worst, float((err / most_off).max()))
        assert worst <= 1, f"{what} {name}: gradient {worst} times the bound"
        ref = T * (1 / S - 1)
        assert abs(g[0, at].item() - ref) <= abs(ref) * (4 * U + R.HALF[z.dtype])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=ids_of)
@pytest.mark.parametrize("T,high", [(1.0, 0.357), (1.0, 1.2), (2.0, 0.21)])
def test_distill_sum_of_a_very_long_row(T, high, dtype):
    """2^27 classes: equal terms, which a float sum rounds the same way once it is large; every lane
    has seen the larger ones before them."""
    n, m = (1 << 27) + 5, 8192
    z = torch.zeros(1, n, dtype=dtype, device="cuda")
    z[0, :m] = high
    most = z[0, 0].item()
    S = m + (n - m) * math.exp(-most / T)
    _check_long_row(z, T, most, S, 17, f"{n} x {high}")


@pytest.mark.parametrize("T", [0.25, 1.0])
@pytest.mark.parametrize("order", ["rising", "falling", "steps", "waves"])
def test_distill_sum_of_a_long_row_in_order(order, T):
    """Logits whose largest moves at every step, now and then, or never."""
    n = (1 << 24) + 3
    j = torch.arange(n, device="cuda", dtype=torch.float64) / n
    z = {"rising": 30 * j, "falling": 30 - 30 * j, "steps": torch.floor(40 * j) * 0.9,
         "waves": torch.sin(200 * j) * 20 * j}[order].float().view(1, -1)
    most, at = z.double().max(1)
    S = torch.exp((z.double() - most) / T).sum().item()
    _check_long_row(z, T, most.item(), S, int(at), f"{order} T={T}")


def test_labels_and_first_scores_part_where_sums_round_alike():
    """Sums of 1 and 1 + 2^-30 are one float: the label is the larger sum's, the first score the
    lower class's."""
    from synth import Forest
    leaf = np.full(3, -1, np.int32)
    model = Forest(n_features=1, n_classes=2, tree_offsets=np.arange(4, dtype=np.int64),
                   feature=np.zeros(3, np.int32), threshold=np.zeros(3, np.float32), left=leaf, right=leaf,
                   value=np.array([1, 1, 2.0 ** -30], np.float32), tree_class=np.array([0, 1, 1], np.int32))
    X = torch.zeros(5, 1, device="cuda")
    with B.Forest(model) as f:
        scores, (values, ids), labels = f.predict(X), f.predict_top(X, 2), f.predict_labels(X)
    assert (scores == 1).all() and (values == 1).all()
    assert ids.tolist() == [[0, 1]] * 5 and labels.tolist() == [1] * 5
    model.value[2] = 2.0 ** -20                    # sums that floats tell apart
    with B.Forest(model) as f:
        ids, labels = f.predict_top(X, 1)[1], f.predict_labels(X)
    assert ids[:, 0].tolist() == labels.tolist() == [1] * 5


def test_negated_views_are_refused():
    """The imaginary part of a conjugate holds the other sign; a row of one element of it looks like
    any other."""
    z = torch.complex(_normal(1, 6, 1), _normal(2, 6, 1)).conj().imag
    assert z.is_neg() and z.shape == (6, 1)
    ids, t = torch.zeros(6, 1, dtype=torch.int32, device="cuda"), torch.zeros(6, 1, device="cuda")
    one, q = torch.ones(1, device="cuda"), torch.ones(1, 4, dtype=torch.int8, device="cuda")
    for call in (lambda: B.top_k(z, 1), lambda: B.distill(z, ids, t), lambda: B.distill(t, ids, z),
                 lambda: B.rmsnorm_q8(z), lambda: B.rmsnorm_q8(t, z[0]), lambda: B.matmul_q8(q, z[0], q, one),
                 lambda: B.distill(t[:1], ids[:1], t[:1], weight=z[0])):
        with pytest.raises(ValueError):
            call()
    values, _ = B.top_k(z.resolve_neg(), 1)
    assert torch.equal(values, z)


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [70001, 140003, 140007])
def test_distill_ends_of_long_rows(width, dtype):
    """The elements past a long row's whole loads, alone or broken, with little or nothing before them."""
    z = torch.full((8, width), -inf, dtype=dtype, device="cuda")
    low = torch.finfo(dtype).min
    z[0, -1] = 3                                  # the only class
    z[1, -1], z[1, 5] = 3, 2
    z[2, -1], z[2, 5] = low, 2
    z[3], z[3, -1] = low, 1
    z[4, -1], z[4, -2] = 1, 1
    z[5, -1], z[5, 5] = nan, 2
    z[6, -1], z[6, 5] = inf, 2
    z[7, -1], z[7, 5] = 2, nan
    ids = torch.full((8, 1), width - 1, dtype=torch.int32, device="cuda")
    t = torch.zeros(8, 1, device="cuda")
    for T in (1.0, 0.5):
        loss, grad = _check_distill(z[:5], ids[:5], t[:5], T, None, f"{width} T={T}")
        assert loss[0] == 0 and loss[3] == 0 and (grad[0] == 0).all()
        loss, grad = B.distill(z[5:], ids[5:], t[5:], T)
        assert torch.isnan(loss).all() and torch.isnan(grad).all()
