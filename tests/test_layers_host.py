"""What the layers and sample refuse, and that they refuse it before any launch: through the C ABI with
addresses that nothing reads, on a machine without a GPU."""
import inspect

import numpy as np
import pytest

import layers_ref as L
import paper_2405_12491_amd as B
from paper_2405_12491_amd import layers, operators

ARG, UNS, DEV = B.BRIDGER_ERR_INVALID_ARGUMENT, B.BRIDGER_ERR_UNSUPPORTED, B.BRIDGER_ERR_DEVICE
NONE = None
A = [(i + 1) << 40 for i in range(10)]     # far addresses
inf, nan = float("inf"), float("nan")
BIG = 1 << 39

EMB = dict(ids=A[0], ldi=3, offsets=A[1], table=A[2], ldt=10, dtype=0, n=5, slots=3, entries=7, features=10, scale=1.0,
           out=A[3], ldo=10, stream=NONE)
EMG = dict(ids=A[0], ldi=3, offsets=A[1], grad=A[2], ldg=10, dtype=0, n=5, slots=3, entries=7, features=10, scale=1.0,
           table=A[3], ldt=10, workspace=A[4], bytes=BIG, stream=NONE)
DRO = dict(x=A[0], ldx=10, residual=A[1], ldr=10, dtype=0, n=5, features=10, p=0.3, seed=A[2], layer=1, out=A[3],
           ldo=10, stream=NONE)
LAN = dict(x=A[0], ldx=10, residual=A[1], ldr=10, weight=A[2], bias=A[3], dtype=0, n=5, features=10, eps=1e-5,
           total=A[4], ldt=10, out=A[5], ldo=10, stats=A[6], stream=NONE)
LNG = dict(grad=A[0], ldg=10, t=A[1], ldt=10, stats=A[2], weight=A[3], grad_total=A[4], lds=10, dtype=0, n=5,
           features=10, dx=A[5], ldd=10, dweight=A[6], dbias=A[7], workspace=A[8], bytes=BIG, stream=NONE)
SAM = dict(logits=A[0], ld=10, dtype=0, n=5, classes=10, u=A[1], temperature=1.0, temperatures=A[2], top_k=3, top_ks=A[3],
           top_p=0.9, top_ps=A[4], min_p=0.1, min_ps=A[5], ids=A[6], logp=A[7], stream=NONE)
FNS = {"bridger_embed": EMB, "bridger_embed_backward": EMG, "bridger_dropout": DRO, "bridger_layer_norm": LAN,
       "bridger_layer_norm_backward": LNG, "bridger_sample": SAM}


def _status(fn, change):
    return getattr(B.load_library(), fn)(*dict(FNS[fn], **change).values())


REFUSED = [
    ("bridger_embed", c, ARG) for c in (
        dict(ids=NONE), dict(table=NONE), dict(out=NONE), dict(dtype=3), dict(dtype=-1), dict(n=-1), dict(n=1 << 31),
        dict(slots=0), dict(slots=-3), dict(entries=0), dict(features=0), dict(scale=inf), dict(scale=nan), dict(ldi=2),
        dict(ldt=9), dict(ldo=9), dict(ids=A[0] + 2), dict(offsets=A[1] + 4), dict(table=A[2] + 2), dict(out=A[3] + 1),
        dict(out=A[2]), dict(out=A[0]), dict(out=A[1] + 24), dict(out=A[2] + 4 * 60), dict(ldt=1 << 62),
        dict(entries=2 ** 31 - 1, ldt=1 << 58))
] + [
    ("bridger_embed_backward", c, ARG) for c in (
        dict(ids=NONE), dict(grad=NONE), dict(table=NONE), dict(workspace=NONE), dict(dtype=5), dict(n=-1), dict(slots=0),
        dict(entries=0), dict(entries=-1), dict(features=0), dict(scale=nan), dict(ldi=2), dict(ldg=9), dict(ldt=9),
        dict(workspace=A[4] + 8), dict(bytes=0), dict(bytes=64), dict(table=A[2]), dict(table=A[0]), dict(table=A[4]),
        dict(workspace=A[2] + 32), dict(grad=A[2] + 2), dict(table=A[3] + 2))
] + [
    ("bridger_embed_backward", dict(n=1 << 30, slots=2, ldi=2), UNS),
    ("bridger_embed_backward", dict(n=2 ** 31 - 1), UNS),
] + [
    ("bridger_dropout", c, ARG) for c in (
        dict(x=NONE), dict(seed=NONE), dict(out=NONE), dict(dtype=3), dict(n=-1), dict(features=0), dict(p=-0.1),
        dict(p=1.0000001), dict(p=nan), dict(layer=-1), dict(ldx=9), dict(ldr=9), dict(ldo=9), dict(x=A[0] + 2),
        dict(residual=A[1] + 1), dict(seed=A[2] + 4), dict(out=A[3] + 2), dict(out=A[0] + 4), dict(out=A[0], ldo=11),
        dict(out=A[1], ldr=12), dict(out=A[2]))
] + [
    ("bridger_layer_norm", c, ARG) for c in (
        dict(x=NONE), dict(out=NONE), dict(dtype=3), dict(n=-1), dict(features=0), dict(eps=-1e-9), dict(eps=nan),
        dict(eps=inf), dict(ldx=9), dict(ldr=9), dict(ldt=9), dict(ldo=9), dict(x=A[0] + 1), dict(weight=A[2] + 2),
        dict(bias=A[3] + 2), dict(stats=A[6] + 2), dict(out=A[0]), dict(out=A[1]), dict(out=A[2]), dict(out=A[4]),
        dict(total=A[0] + 4), dict(total=A[0], ldt=12), dict(stats=A[5] + 40), dict(stats=A[3]))
] + [
    ("bridger_layer_norm_backward", c, ARG) for c in (
        dict(grad=NONE), dict(t=NONE), dict(stats=NONE), dict(dx=NONE, dweight=NONE, dbias=NONE), dict(dtype=3),
        dict(n=-1), dict(features=0), dict(ldg=9), dict(ldt=9), dict(lds=9), dict(ldd=9), dict(workspace=NONE),
        dict(bytes=0), dict(bytes=399), dict(workspace=A[8] + 4), dict(dx=A[0]), dict(dx=A[1]), dict(dx=A[4]),
        dict(dweight=A[3]), dict(dbias=A[6]), dict(dx=A[8]), dict(dweight=A[8] + 16), dict(grad=A[0] + 2),
        dict(stats=A[2] + 2), dict(dweight=A[6] + 1))
] + [
    ("bridger_sample", c, ARG) for c in (
        dict(logits=NONE), dict(u=NONE), dict(ids=NONE), dict(dtype=3), dict(n=-1), dict(n=1 << 31), dict(classes=0),
        dict(ld=9), dict(temperature=-0.1), dict(temperature=nan), dict(temperature=inf), dict(temperature=1e7),
        dict(top_k=-1), dict(top_p=-0.1), dict(top_p=1.1), dict(top_p=nan), dict(min_p=-0.1), dict(min_p=1.1),
        dict(min_p=nan), dict(logits=A[0] + 2), dict(u=A[1] + 2), dict(temperatures=A[2] + 1), dict(top_ks=A[3] + 1),
        dict(top_ps=A[4] + 2), dict(min_ps=A[5] + 3), dict(ids=A[6] + 2), dict(logp=A[7] + 2), dict(ids=A[0]),
        dict(logp=A[1] + 16), dict(logp=A[6]), dict(ids=A[3]))
]


@pytest.mark.parametrize("case", range(len(REFUSED)))
def test_refused(case):
    fn, change, status = REFUSED[case]
    assert _status(fn, change) == status, (fn, change)
    assert B.bridger_last_error(), (fn, change)


SOUND = [("bridger_embed", c) for c in (dict(), dict(offsets=NONE), dict(n=1, ldi=0), dict(ids=A[0], table=A[0] + 4096),
                                        dict(scale=-2.0))] + [
    ("bridger_embed_backward", c) for c in (dict(), dict(offsets=NONE), dict(n=0, ids=NONE, grad=NONE, offsets=NONE))] + [
    ("bridger_dropout", c) for c in (dict(), dict(residual=NONE), dict(out=A[0]), dict(out=A[1]), dict(p=0.0), dict(p=1.0),
                                     dict(layer=2 ** 31 - 1), dict(ldx=20, out=A[0] + 40, ldo=20))] + [
    ("bridger_layer_norm", c) for c in (dict(), dict(residual=NONE, total=NONE, weight=NONE, bias=NONE, stats=NONE),
                                        dict(total=A[0]), dict(total=A[1]), dict(eps=0.0))] + [
    ("bridger_layer_norm_backward", c) for c in (
        dict(), dict(weight=NONE, grad_total=NONE), dict(dx=NONE), dict(dweight=NONE),
        dict(dweight=NONE, dbias=NONE, workspace=NONE, bytes=0), dict(n=0, grad=NONE, t=NONE, stats=NONE, workspace=NONE))] + [
    ("bridger_sample", c) for c in (dict(), dict(temperatures=NONE, top_ks=NONE, top_ps=NONE, min_ps=NONE, logp=NONE),
                                    dict(temperature=0.0, top_k=0, top_p=0.0, min_p=1.0), dict(u=A[2]))]


@pytest.mark.parametrize("case", range(len(SOUND)))
def test_sound_arguments_pass_the_checks(case):
    import torch
    if torch.cuda.is_available():
        pytest.skip("these addresses must not reach a GPU")
    fn, change = SOUND[case]
    assert _status(fn, change) == DEV, (fn, change, B.bridger_last_error())


def test_no_rows_need_no_device():
    for fn in ("bridger_embed", "bridger_dropout", "bridger_layer_norm", "bridger_sample"):
        assert _status(fn, dict(n=0)) == B.BRIDGER_OK and B.bridger_last_error() == ""
    assert _status("bridger_layer_norm_backward", dict(n=0, dweight=NONE, dbias=NONE)) == B.BRIDGER_OK


def test_workspace_sizes():
    f, g = B.bridger_embed_backward_workspace, B.bridger_layer_norm_backward_workspace
    for bad in ((-1, 1, 5, 5), (1 << 31, 1, 5, 5), (5, 0, 5, 5), (5, 1, 0, 5), (5, 1, 5, 0), (1 << 30, 2, 5, 5)):
        assert f(*bad) == 0, bad
    for bad in ((-1, 5, 0), (5, 0, 0), (5, 5, 3), (0, 5, 0)):
        assert g(*bad) == 0, bad
    # a pair takes 8 bytes, twice where many are sorted; two sums of 4 bytes an element for each block
    for n, k, e, w in ((1, 1, 1, 1), (16384, 1, 50257, 1024), (16385, 1, 50257, 7), (5000, 100, 51100, 64),
                       (2 ** 31 - 1, 1, 2 ** 31 - 1, 4), (100, 1, 2 ** 31 - 1, 8)):
        pairs = n * k
        blocks = -(-pairs // 128)
        assert f(n, k, e, w) >= 8 * pairs + 8 * blocks * w, (n, k, e, w)
        assert f(n, k, e, w) <= 64 * pairs + 8 * (pairs // 16 + 1) * w + (1 << 20), (n, k, e, w)
        assert f(n, k, e, w) % 16 == 0
    for n, w in ((1, 1), (8192, 4096), (10 ** 6, 28), (3, 2 ** 31 - 1)):
        assert g(n, w, 0) % (8 * w) == 0 and 8 * w <= g(n, w, 0) <= 2048 * 8 * w


def test_cpu_tensors_are_refused():
    import torch
    x, u = torch.zeros(3, 8), torch.zeros(3)
    ids = torch.zeros(3, 2, dtype=torch.int32)
    seed = torch.zeros(2, dtype=torch.int64)
    for call in (lambda: B.embed(ids, x), lambda: B.embed(ids[:, 0], x), lambda: B.embed([1], x), lambda: B.embed(None, x),
                 lambda: B.embed_grad(ids, x, 4), lambda: B.dropout(x, 0.5, seed), lambda: B.dropout([[1.0]], 0.5, seed),
                 lambda: B.layer_norm(x), lambda: B.layer_norm_grad(x, x, x[:, :3]), lambda: B.sample(x, u),
                 lambda: B.layer_norm(x.requires_grad_()), lambda: B.embed(ids, x), lambda: B.dropout(x, 0.5, seed)):
        with pytest.raises(TypeError):
            call()


def test_tangents_are_refused():
    """What the layers differentiate gives no tangents: inputs and outputs that have one are refused, in
    grad mode and without; tensors without one are as ever."""
    import torch
    import torch.autograd.forward_ad as fa
    x, w, seed = torch.zeros(3, 8), torch.zeros(8), torch.zeros(2, dtype=torch.int64)
    ids = torch.zeros(3, 2, dtype=torch.int32)
    calls = [lambda d, v: B.embed(ids, d), lambda d, v: B.embed(ids, x, out=d), lambda d, v: B.dropout(d, 0.5, seed),
             lambda d, v: B.dropout(x, 0.5, seed, residual=d), lambda d, v: B.dropout(x, 0.5, seed, out=d),
             lambda d, v: B.layer_norm(d), lambda d, v: B.layer_norm(x, v), lambda d, v: B.layer_norm(x, w, v),
             lambda d, v: B.layer_norm(x, residual=d), lambda d, v: B.layer_norm(x, out=d),
             lambda d, v: B.layer_norm(x, total=d), lambda d, v: B.layer_norm(x, stats=d)]
    with fa.dual_level():
        d, v = fa.make_dual(x, torch.ones(3, 8)), fa.make_dual(w, torch.ones(8))
        for i, call in enumerate(calls):
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(NotImplementedError, match="tangent"):
                    call(d, v)
                    pytest.fail(f"call {i} was not refused")
            with pytest.raises(TypeError, match="CUDA"):
                call(x, w)
    with pytest.raises(TypeError, match="CUDA"):
        B.embed(ids, x)


def test_raw_calls_report_their_errors():
    with pytest.raises(B.BridgerError, match="n_slots") as e:
        B.bridger_embed(A[0], 3, None, A[2], 10, 0, 5, 0, 7, 10, 1.0, A[3], 10)
    assert e.value.status == ARG
    with pytest.raises(B.BridgerError, match="workspace is too small"):
        B.bridger_embed_backward(A[0], 3, None, A[2], 10, 0, 5, 3, 7, 10, 1.0, A[3], 10, A[4], 16)
    with pytest.raises(B.BridgerError, match="p must lie"):
        B.bridger_dropout(A[0], 10, None, 0, 0, 5, 10, 2.0, A[2], 0, A[3], 10)
    with pytest.raises(B.BridgerError, match="eps"):
        B.bridger_layer_norm(A[0], 10, None, 0, None, None, 0, 5, 10, -1.0, None, 0, A[5], 10, None)
    with pytest.raises(B.BridgerError, match="no output"):
        B.bridger_layer_norm_backward(A[0], 10, A[1], 10, A[2], None, None, 0, 0, 5, 10, None, 0, None, None, None, 0)
    with pytest.raises(B.BridgerError, match="temperature"):
        B.bridger_sample(A[0], 10, 0, 5, 10, A[1], -1.0, None, 0, None, 1.0, None, 0.0, None, A[6], None)


def test_every_raw_function_has_its_entry_point():
    lib = B.load_library()
    for name, types in list(layers._ARGTYPES.items()) + list(operators._ARGTYPES.items()):
        assert len(getattr(lib, name).argtypes) == len(types)
        assert len(inspect.signature(getattr(B, name)).parameters) == len(types), name
    for name, types in layers._SIZES.items():
        assert len(inspect.signature(getattr(B, name)).parameters) == len(types), name


def test_random_words_known_answers():
    """The published test vectors of Philox4x32-10 (Random123's kat_vectors)."""
    for counter, key, want in (
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        got = L.random_words(*counter, *key)
        assert tuple(int(v) for v in got) == want


def test_reference_of_sample():
    """The definition on rows that can be drawn by hand."""
    z = np.log([1.0, 4.0, 2.0, 3.0])
    assert [L.sample_row(z, u)[0] for u in (0.0, 0.05, 0.15, 0.55, 0.65, 0.75, 0.99)] == [0, 0, 1, 2, 2, 3, 3]
    assert sorted(L.sample_row(z, 0.5, top_k=2)[2]) == [1, 3]
    assert sorted(L.sample_row(z, 0.5, top_p=0.65)[2]) == [1, 3]
    assert sorted(L.sample_row(z, 0.5, top_p=0.75)[2]) == [1, 2, 3]
    assert sorted(L.sample_row(z, 0.5, min_p=0.6)[2]) == [1, 3]
    assert L.sample_row([-np.inf, np.nan], 0.5)[0] == -1
    assert L.sample_row([1.0, 1.0, 0.0], 0.9, temperature=0.0)[0] == 0
