"""sample on the GPU against its definition in 64 bits (layers_ref.sample_row): widths from one class to
long rows, every cut alone and with others, equal scores, masked and broken rows, parameters by row."""
import math

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


def _logits(seed, n, c, dtype, scale=3.0):
    return (torch.randn(n, c, generator=_gen(seed), device="cuda") * scale).to(dtype)


def _u(seed, n):
    return torch.rand(n, generator=_gen(seed), device="cuda")


def _check(z, u, what="", undecided=1, **how):
    """Ids equal, but for draws nearer to another class than sums in double tell apart (`undecided` rows at
    most); logp off by its rounding to float, and by that of the weights and sums in double."""
    ids, logp = B.sample(z, u, **how)
    zn, un, got, lp = np64(z), np64(u), ids.cpu().numpy(), np64(logp)
    per = {k: np64(v) if torch.is_tensor(v) else [v] * len(zn) for k, v in how.items()}
    sure = 0
    for r in range(len(zn)):
        args = {k: v[r] for k, v in per.items()}
        args["top_k"] = int(args.get("top_k", 0))
        want, ref, stay, gap = L.sample_row(zn[r], un[r], **args)
        if gap < 1e-11:
            continue
        sure += 1
        assert got[r] == want, f"{what} row {r}: {got[r]}, not {want} ({args})"
        if np.isinf(ref):
            assert lp[r] == ref
        else:
            assert abs(lp[r] - ref) <= R.U * abs(ref) + 1e-11, f"{what} row {r}: {lp[r]}, not {ref}"
    assert sure >= len(zn) - undecided, what
    return ids, logp


WIDTHS = [1, 2, 3, 5, 8, 10, 33, 64, 100, 257, 512, 513, 1000, 1025, 2048, 2049, 4097, 8191, 8195, 16385, 32769,
          50_257, 65_537, 131_077, 150_001]
WAYS = [dict(), dict(temperature=0.4), dict(temperature=2.5, top_k=5), dict(top_k=1), dict(top_k=40, top_p=0.8),
        dict(top_p=0.9), dict(top_p=0.3, temperature=1.5), dict(min_p=0.05), dict(top_p=0.95, min_p=0.02),
        dict(top_k=200, top_p=0.97, min_p=0.001, temperature=0.9), dict(temperature=0.0), dict(top_p=0.0),
        dict(min_p=1.0), dict(top_k=2 ** 31 - 1)]


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", WIDTHS)
def test_sample(width, dtype):
    n = 4 if width > 10_000 else 19
    z, u = _logits(width, n, width, dtype), _u(width + 1, n)
    for i, how in enumerate(WAYS):
        _check(z, u, f"{how}", **how)


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [700, 3000, 20_000, 140_000])
def test_sample_more_than_lds_holds(width, dtype):
    """Flat rows, whose cuts lie far down: top_p of many classes, top_k above what is sorted."""
    z, u = _logits(width, 3, width, dtype, scale=0.05), _u(3, 3)
    for how in (dict(top_p=0.7), dict(top_p=0.999), dict(top_k=width // 2), dict(top_k=width - 1, top_p=0.5),
                dict(top_k=2500, top_p=0.9, min_p=0.9), dict(top_k=2048), dict(top_k=2049), dict(top_k=1025)):
        _check(z, u, f"{how}", **how)


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [2, 9, 64, 600, 5000, 40_000, 140_000])
def test_sample_equal_scores(width, dtype):
    """Ties are kept in the order of their classes, to the class."""
    j = torch.arange(width, device="cuda", dtype=torch.float32)
    rows = [torch.zeros(width, device="cuda"), (j % 2), -(j % 3), torch.where(j % 64 == 3, 2.0, -2.0),
            torch.where(j % 2 == 0, 0.0, -0.0), torch.where(j == width - 1, 1.0, 0.0), torch.floor(j * 8 / width)]
    z = torch.stack(rows).to(dtype)
    u = _u(width, len(rows))
    for how in (dict(), dict(top_k=width // 2 + 1), dict(top_p=0.5), dict(top_p=0.37, top_k=width // 3 + 1),
                dict(min_p=1.0), dict(top_k=7), dict(top_p=1e-9), dict(temperature=0.0)):
        _check(z, u, f"{how}", **how)
    for last in (0.0, 1 - 2.0 ** -24):
        for how in (dict(), dict(top_k=width // 2 + 1), dict(top_p=0.5)):
            _check(z, torch.full_like(u, last), f"{how} u={last}", **how)


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [1, 3, 50, 700, 9000, 70_000, 140_000])
def test_sample_masked_and_broken(width, dtype):
    low = torch.finfo(dtype).min
    z = _logits(1, 12, width, dtype)
    z[0] = -inf
    z[1] = nan
    z[2] = inf
    z[3, ::2] = nan
    z[4, 1:] = -inf
    z[5, :-1] = nan
    z[6, ::3] = -inf
    z[7, -1] = inf
    z[8] = low
    z[9, 1:] = low
    z[10, :-1] = -inf
    z[11, ::2] = inf
    u = _u(2, 12)
    for how in (dict(), dict(top_k=3), dict(top_p=0.6), dict(min_p=0.1), dict(temperature=0.0),
                dict(top_k=100, top_p=0.99, min_p=0.01, temperature=0.5)):
        ids, logp = _check(z, u, f"{how}", **how)
        assert ids[:2].tolist() == [-1, -1] and bool((logp[:2] == -inf).all())
        # a masked class is never drawn
        at = ids[2:].long()
        ok = at >= 0
        picked = z[2:].gather(1, at.clamp(min=0)[:, None])[:, 0]
        assert bool((picked[ok] > -inf).all())


@pytest.mark.parametrize("how", [dict(), dict(top_k=6), dict(top_p=0.85), dict(min_p=0.05)])
def test_sample_shares(how):
    """Evenly spread random numbers give each class its share of the rows, to one row."""
    n = 10_000
    z = _logits(5, 1, 40, torch.float32)
    u = (torch.arange(n, device="cuda") + 0.5) / n
    ids, logp = B.sample(z.expand(n, 40).contiguous(), u, **how)
    _, _, stay, _ = L.sample_row(np64(z)[0], 0.5, **how)
    w = np.exp(np64(z)[0, stay] - np64(z)[0, stay].max())
    share = np.zeros(40)
    share[stay] = w / w.sum()
    count = np.bincount(ids.cpu().numpy(), minlength=40)
    assert np.abs(count - n * share).max() <= 1.01
    assert np.allclose(np.exp(np64(logp)), share[ids.cpu().numpy()], rtol=1e-6)
    assert bool((ids[1:] >= ids[:-1]).all())      # the draw runs in the order of the classes


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [5, 300, 5000])
def test_sample_own_parameters(width, dtype):
    n = 40
    z, u = _logits(1, n, width, dtype), _u(2, n)
    g = _gen(3)
    how = dict(temperature=torch.rand(n, generator=g, device="cuda") * 2,
               top_k=torch.randint(-2, 80, (n,), generator=g, device="cuda", dtype=torch.int32),
               top_p=torch.rand(n, generator=g, device="cuda") * 1.2,
               min_p=torch.rand(n, generator=g, device="cuda") * 0.2 - 0.05)
    how["temperature"][:5] = torch.tensor([0.0, -1.0, nan, 1e9, 1e-7], device="cuda")
    how["top_p"][5:8] = torch.tensor([-0.5, 1.0, 2.0], device="cuda")
    how["min_p"][8:10] = torch.tensor([5.0, 1.0], device="cuda")
    _check(z, u, **how)
    none = dict(top_p=torch.full((n,), nan, device="cuda"), min_p=torch.full((n,), nan, device="cuda"))
    assert torch.equal(B.sample(z, u, **none)[0], B.sample(z, u)[0])
    # one tensor among numbers
    _check(z, u, temperature=0.7, top_k=how["top_k"], min_p=0.01)
    same = torch.full((n,), 9, dtype=torch.int32, device="cuda")
    assert torch.equal(B.sample(z, u, top_k=same)[0], B.sample(z, u, top_k=9)[0])


def test_sample_random_numbers_outside_their_range():
    z = _logits(1, 6, 100, torch.float32)
    u = torch.tensor([-1.0, nan, 1.0, 7.0, inf, -inf], device="cuda")
    inside = torch.tensor([0.0, 0.0, 1 - 2.0 ** -24, 1 - 2.0 ** -24, 1 - 2.0 ** -24, 0.0], device="cuda")
    assert torch.equal(B.sample(z, u)[0], B.sample(z, inside)[0])


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width,gap,lead", [(5, 1, 1), (65, 3, 1), (1000, 7, 3), (5003, 1, 0), (140_001, 2, 5)])
def test_sample_strided_and_given_outputs(width, gap, lead, dtype):
    n = 7
    z, u = _logits(1, n, width, dtype), _u(2, n)
    buf = torch.full((n * (width + gap) + lead + 3,), 100.0, dtype=dtype, device="cuda")
    sz = buf[lead:lead + n * (width + gap)].view(n, width + gap)[:, :width]
    sz.copy_(z)
    ids, logp = torch.full((n + 2,), 9, dtype=torch.int32, device="cuda"), torch.full((n + 2,), 9.0, device="cuda")
    for how in (dict(), dict(top_k=20), dict(top_p=0.9), dict(top_p=0.9, temperature=30.0)):
        want = B.sample(z, u, **how)
        got = B.sample(sz, u, ids=ids[1:-1], logp=logp[1:-1], **how)
        assert got[0].data_ptr() == ids[1:].data_ptr()
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    assert ids[0] == 9 and ids[-1] == 9 and logp[0] == 9 and logp[-1] == 9
    only = torch.full((n,), 9, dtype=torch.int32, device="cuda")
    code = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[dtype]
    B.bridger_sample(sz.data_ptr(), sz.stride(0), code, n, width, u.data_ptr(), 30.0, None, 0, None, 0.9, None, 0.0,
                     None, only.data_ptr(), None, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(only, want[0])


def test_sample_no_rows():
    ids, logp = B.sample(torch.empty(0, 10, device="cuda"), torch.empty(0, device="cuda"))
    assert ids.shape == logp.shape == (0,) and ids.dtype == torch.int32


@pytest.mark.parametrize("n", [2, 63, 1000, 20_011])
def test_sample_rows(n):
    z, u = _logits(n, n, 12, torch.float32), _u(n, n)
    ids, _ = B.sample(z, u, temperature=0.8)
    w = torch.softmax(z.double() / 0.8, 1)
    at = (torch.cumsum(w, 1) <= u.double()[:, None]).sum(1).clamp(max=11)
    # sums of twelve in double: a draw within 1e-12 of a border may go either way
    near = (torch.cumsum(w, 1) - u.double()[:, None]).abs().min(1).values < 1e-12
    assert bool(((ids == at) | near).all())


def test_sample_extreme_temperatures():
    z, u = _logits(1, 9, 300, torch.float32), _u(2, 9)
    for T in (1e-6, 1e-5, 1e-3, 1e3, 1e6):
        _check(z, u, f"{T}", temperature=T)
        _check(z * 1e30, u, f"{T}, huge scores", temperature=T)


def test_sample_agrees_with_top_k():
    """A temperature of 0 takes top_k's first class; what is drawn is among the top_k."""
    z, u = _logits(1, 50, 3000, torch.bfloat16, scale=1.0), _u(2, 50)
    _, top = B.top_k(z, 20)
    assert torch.equal(B.sample(z, u, temperature=0.0)[0], top[:, 0])
    ids, _ = B.sample(z, u, top_k=20)
    assert bool((top == ids[:, None]).any(1).all())


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [257, 300, 500, 1000, 1025, 5000, 50_257, 140_000])
def test_sample_cuts_below_what_is_ranked(width, dtype):
    """More classes stay than are ranked by counting: by top_p, by min_p, and by the one although the other
    would leave more; whole numbers (many equal scores at the cut), masked rows, far ranges."""
    n = 8 if width > 10_000 else 60
    z, u = _logits(width + 7, n, width, dtype, scale=2.0), _u(width + 8, n)
    z[1] = z[1].round()
    z[2, ::2] = -inf
    z[3, 1:] -= 60.0
    z[4] *= 20.0
    z[5] = torch.where(z[5] > 0, 3.0, -3.0).to(dtype)
    z[6, :width // 2] = nan
    z[7] = z[7] * 0.001 + 40.0
    for how in (dict(temperature=1.5, min_p=0.001), dict(temperature=3.0, min_p=0.01),
                dict(temperature=1.5, top_p=0.95), dict(temperature=2.0, top_p=0.999, min_p=0.02),
                dict(temperature=4.0, top_p=0.7, min_p=1e-4), dict(temperature=50.0, top_p=0.4),
                dict(temperature=0.05, top_p=0.9999999), dict(top_p=1e-6, min_p=1e-6),
                dict(temperature=1e6, top_p=0.5), dict(temperature=1e-5, top_p=0.5)):
        # at 1e-5 the classes of the largest score weigh 1 and all others nearly nothing: with an even
        # number of them the weight before one is top_p of all, exactly
        top = (z == z.nan_to_num(-inf).amax(1, keepdim=True)).sum(1)
        halves = int((top % 2 == 0).sum()) if how.get("temperature") == 1e-5 else 0
        _check(z, u, f"{how}", undecided=1 + halves, **how)


def test_sample_shares_of_bins():
    """Cuts by top_p at each class in turn, of scores that are spread evenly, stay where the definition has
    them."""
    n, c = 700, 900
    z = (torch.arange(c, device="cuda") * -0.004).expand(n, c).contiguous()
    p = (torch.arange(n, device="cuda") + 0.5) / n
    _check(z, _u(1, n), top_p=p)
    _check(z.flip(1).contiguous(), _u(1, n), top_p=p, min_p=0.2)


@pytest.mark.parametrize("own", [False, True])
def test_sample_top_k_near_its_largest(own):
    """top_k within a step of 2^31, of a row with more classes, nearly all of them masked."""
    n = 2 ** 31 - 1
    z = torch.full((1, n), -inf, dtype=torch.bfloat16, device="cuda")
    at = torch.cat([torch.randint(0, n, (97,), generator=_gen(1), device="cuda"), torch.tensor([0, n - 1], device="cuda")])
    z[0, at] = _logits(2, 1, 99, torch.bfloat16)[0]
    some = torch.unique(at)
    scores = np64(z[0, some])
    for k in (n - 15, n - 1, n // 2 + 3):
        for u in (0.0, 0.3, 0.9999):
            top_k = torch.tensor([k], dtype=torch.int32, device="cuda") if own else k
            ids, logp = B.sample(z, torch.tensor([u], device="cuda"), temperature=1.3, top_k=top_k, top_p=0.9)
            want, ref, _, gap = L.sample_row(scores, float(np.float32(u)), temperature=1.3, top_k=k, top_p=0.9)
            assert gap > 1e-11
            assert int(ids) == int(some[want]) and abs(float(logp) - ref) <= R.U * abs(ref) + 1e-11


def _check_consistent(z, u, what="", **how):
    """Every row's class and logp are those of sums that are off by 1e-11 of all at most, near a border too."""
    ids, logp = B.sample(z, u, **how)
    zn, un, got, lp = np64(z), np64(u), ids.cpu().numpy(), np64(logp)
    top_k, p, T, m = (how.get(k, d) for k, d in (("top_k", 0), ("top_p", 1.0), ("temperature", 1.0), ("min_p", 0.0)))
    for r in range(len(zn)):
        cls = np.flatnonzero(zn[r] > -np.inf)
        cls = cls[np.argsort(-zn[r, cls], kind="stable")]
        v = zn[r, cls[:top_k or None]]
        w = np.exp((v - v[0]) / T)
        before = np.concatenate([[0.0], np.cumsum(w)])
        limit, doubt = p * before[-1], 1e-11 * before[-1]
        # the classes that may be the last to stay, and what stays for the fewest and the most
        fewest, most = (max(1, int((before[:-1] < limit + d).sum())) for d in (-doubt, doubt)) if p < 1 else (len(w),) * 2
        above = int((v >= v[0] + T * np.log(m)).sum()) if m > 0 else len(w)
        rank = np.flatnonzero(cls == got[r])
        assert len(rank) == 1 and rank[0] < min(most, above), f"{what} row {r}: class {got[r]} does not stay"
        fits = []
        for stay in sorted({min(s, above) for s in (fewest, max(fewest, rank[0] + 1), most)}):
            if stay > rank[0]:
                order = np.argsort(cls[:stay])
                sums = np.cumsum(w[:stay][order])
                at = int(np.flatnonzero(cls[:stay][order] == got[r])[0])
                begin, target = sums[at] - w[rank[0]], un[r] * sums[-1]
                fits.append(begin - doubt <= target <= sums[at] + doubt and
                            abs(lp[r] - np.log(w[rank[0]] / sums[-1])) <= R.U * abs(lp[r]) + 1e-10)
        assert any(fits), f"{what} row {r}: class {got[r]}, logp {lp[r]}"


@pytest.mark.parametrize("dtype", TYPES, ids=ids_of)
@pytest.mark.parametrize("width", [257, 1025, 5000, 50_257, 140_000])
def test_sample_near_borders(width, dtype):
    """Halves that are exact but for rounding, and draws at a class's edge: one of the two neighbours."""
    z = _logits(width + 7, 8, width, dtype, scale=2.0)
    z[1] = z[1].round()
    z[2, ::2] = -inf
    z[3, :width // 2] = z[3, 0]
    u = _u(width, 8)
    u[::3] = 0.5
    for how in (dict(temperature=1e-5, top_p=0.5), dict(temperature=1e6, top_p=0.5), dict(top_p=0.5, temperature=50.0),
                dict(temperature=1e6, top_k=width // 2 * 2, top_p=0.25), dict(temperature=1e6), dict(top_p=0.5, min_p=0.3)):
        _check_consistent(z, u, f"{how}", **how)


@pytest.mark.parametrize("width,head", [(9000, 3000), (20_000, 2500), (50_257, 4000)])
def test_sample_cut_at_the_end_of_a_cluster(width, head):
    """A share of the classes stands close together, and top_p is their share of the mass, to the last bits:
    they stay, and one more at most."""
    rng = np.random.default_rng(width)
    for turn in range(8):
        z = rng.uniform(-1.0, 0.0, width).astype(np.float32)
        place = rng.permutation(width)[:head]
        z[place] = np.float32(4.0) + np.float32(2.0 ** -21) * rng.integers(0, 1500 * (turn + 1), head).astype(np.float32)
        w = np.exp(z.astype(np.float64) - z.max())
        p = math.fsum(w[place]) / math.fsum(w)
        rows = torch.from_numpy(z).cuda().expand(3, width).contiguous()
        u = torch.tensor([0.1, 0.5, 0.999], device="cuda")
        for ulps in range(-4, 5):
            _check_consistent(rows, u, f"{turn} {ulps}", top_p=p + ulps * np.spacing(p))
