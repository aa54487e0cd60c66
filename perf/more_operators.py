"""The work of the row operators with which a student of a forest is trained and answers: a lookup of
leaves or tokens in a table and its gradient, layer norm, dropout, and a draw from class scores.

A case is a dict of plain values: ``op``, its sizes (``rows``, ``width`` of a row) and the type
``dtype`` of the rows.  ``run`` computes it with elementary torch operations, or, when ``own`` is set,
with the library's kernels.

* "embed": ``slots`` ids a row, looked up in a table of ``entries`` rows and added up (``way``
  "lookup"), or the table's gradient (``way`` "gradient").  More than one slot: the leaves of a forest,
  each tree with its own part of the table.
* "layer_norm": with the sum of a ``residual`` first; the norm alone (``way`` "forward") or with
  every gradient (``way`` "step").
* "dropout": a share ``p`` of the elements to zero, ``residual`` added after; forward, or "step" with
  the gradient.
* "sample": a class of every row, drawn with ``temperature`` among its ``top_k`` largest scores (0: all),
  the share ``top_p`` of their mass and those of at least ``min_p`` times the largest's probability;
  ``per_row``: each row has parameters of its own.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
EPS = 1e-5
DEV = "cuda"


def listed():
    return [
        # serving one token
        dict(name="embed_one_token", op="embed", way="lookup", rows=1, slots=1, entries=128_000,
             width=4_096, dtype="bf16"),
        # a training step's tokens, some of them padding
        dict(name="embed_tokens_16k", op="embed", way="lookup", rows=16_384, slots=1,
             entries=50_257, width=4_096, dtype="bf16"),
        # the leaves of a random forest of 100 trees of depth 8
        dict(name="embed_leaves_16k", op="embed", way="lookup", rows=16_384, slots=100,
             entries=51_100, width=64, dtype="fp32"),
        # the table's gradient of a training step: few frequent tokens, many rare ones
        dict(name="embed_grad_tokens_16k", op="embed", way="gradient", rows=16_384, slots=1,
             entries=50_257, width=1_024, dtype="bf16"),
        # and of the forest's leaves: thousands of rows a leaf
        dict(name="embed_grad_leaves_16k", op="embed", way="gradient", rows=16_384, slots=100,
             entries=51_100, width=64, dtype="fp32"),
        # serving one row
        dict(name="norm_one_row", op="layer_norm", way="forward", rows=1, width=4_096,
             residual=True, dtype="bf16"),
        # a training step inside a deep model
        dict(name="norm_step_8k", op="layer_norm", way="step", rows=8_192, width=4_096,
             residual=True, dtype="bf16"),
        # a training step on a table's few features
        dict(name="norm_table_1m", op="layer_norm", way="step", rows=1_000_000, width=28,
             residual=False, dtype="fp32"),
        # a block's output in training, added to the running sum
        dict(name="dropout_batch_8k", op="dropout", way="forward", rows=8_192, width=8_192, p=0.1,
             residual=True, dtype="bf16"),
        # a training step on odd rows
        dict(name="dropout_step_100k", op="dropout", way="step", rows=100_000, width=347, p=0.3,
             residual=False, dtype="fp32"),
        # serving one sequence
        dict(name="sample_one_row", op="sample", rows=1, width=128_000, temperature=0.8, top_k=50,
             top_p=0.9, min_p=0.0, per_row=False, dtype="bf16"),
        # a batch of requests, each with its own parameters
        dict(name="sample_batch_512", op="sample", rows=512, width=50_257, temperature=1.0, top_k=0,
             top_p=0.95, min_p=0.02, per_row=True, dtype="fp32"),
    ]


def _loguniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["embed", "embed", "embed", "layer_norm", "layer_norm", "dropout", "sample",
                     "sample"])
    c = dict(op=op, dtype=rng.choice(["fp32", "bf16", "bf16", "fp16"]))
    if op == "embed":
        width = _loguniform(rng, 8, 8_192)
        c.update(way=rng.choice(["lookup", "gradient"]), width=width)
        entries = _loguniform(rng, 64, min(200_000, 100_000_000 // width))
        if rng.random() < 0.5:
            rows, slots = _loguniform(rng, 1, min(65_536, max(1, 64_000_000 // width))), 1
        else:
            slots = _loguniform(rng, 2, min(500, entries // 4))
            rows = _loguniform(rng, 1, max(1, min(65_536, 100_000_000 // (slots * width))))
        c.update(rows=rows, slots=slots, entries=entries)
    elif op in ("layer_norm", "dropout"):
        width = _loguniform(rng, 4, 20_000)
        if rng.random() < 0.4:  # as models have them: whole multiples
            width = (width + 63) // 64 * 64
        c.update(way=rng.choice(["forward", "step"]), width=width, residual=rng.random() < 0.5,
                 rows=_loguniform(rng, 1, min(1_000_000, 30_000_000 // width)))
        if op == "dropout":
            c.update(p=rng.choice([0.05, 0.1, 0.2, 0.3, 0.5]))
    else:
        # from a forest's classes to a vocabulary, from one row to a large batch
        width = _loguniform(rng, 2, 160_000)
        c.update(width=width, rows=_loguniform(rng, 1, max(1, min(50_000, 25_000_000 // width))),
                 temperature=rng.choice([0.3, 0.7, 1.0, 1.0, 1.5]),
                 top_k=rng.choice([0, 0, 1, 10, 50, 200]), top_p=rng.choice([1.0, 0.5, 0.9, 0.95]),
                 min_p=rng.choice([0.0, 0.0, 0.01, 0.1]), per_row=rng.random() < 0.3)
    return c


# ------------------------------------------------------------------------------ inputs
def _normal(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def _uniform(gen, *shape):
    return torch.rand(*shape, generator=gen, device=DEV)


def _embed_inputs(s, gen, n, w, dt):
    k, entries = s["slots"], s["entries"]
    if k == 1:
        # token ids as texts have them: a token's share falls with its number
        ids = (torch.exp(_uniform(gen, n, 1).double() * math.log(entries)) - 1).long()
        pad = _uniform(gen, n, 1) < 1 / 32
        s["ids"] = torch.where(pad, -1, ids.clamp_(0, entries - 1)).to(torch.int32)[:, 0].contiguous()
        s["offsets"] = None
    else:
        # trees of different sizes, whose leaves hold different shares of the rows
        size = 0.5 + _uniform(gen, k).double()
        cut = torch.cumsum(1 + size / size.sum() * (entries - k - 1), 0).long().clamp_(max=entries)
        cut[-1] = entries
        s["offsets"] = torch.cat([cut.new_zeros(1), cut])
        nodes = s["offsets"][1:] - s["offsets"][:-1]
        ids = (_uniform(gen, n, k).double() ** 1.5 * nodes).long()
        s["ids"] = torch.minimum(ids, nodes - 1).to(torch.int32)
    s["scale"] = 1.0 / k if k > 1 else math.sqrt(w)
    if s["way"] == "lookup":
        s["table"] = (_normal(gen, entries, w) / math.sqrt(w)).to(dt)
    else:
        s["grad"] = (_normal(gen, n, w) * 0.01).to(dt)


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    op, n, w, dt = case["op"], case["rows"], case["width"], TYPES[case["dtype"]]
    s = dict(case)
    if op == "embed":
        _embed_inputs(s, gen, n, w, dt)
        return s
    if op == "sample":
        z = _normal(gen, n, w)
        # class scores of a trained model: most low, a few that stand out
        s["logits"] = (2.0 * z + 0.3 * z.abs() * z).to(dt)
        s["u"] = _uniform(gen, n)
        if case["per_row"]:
            s["temperature"] = (0.5 + _uniform(gen, n)) * case["temperature"]
            s["top_k"] = torch.full((n,), case["top_k"], dtype=torch.int32, device=DEV)
            s["top_p"] = (case["top_p"] - 0.1 * _uniform(gen, n)) if case["top_p"] < 1 else \
                torch.ones(n, device=DEV)
            s["min_p"] = case["min_p"] * _uniform(gen, n)
        return s
    s["x"] = _normal(gen, n, w).to(dt)
    s["residual"] = _normal(gen, n, w).to(dt) if case["residual"] else None
    step = case["way"] == "step"
    if op == "layer_norm":
        s["weight"] = (1 + 0.2 * _normal(gen, w)).to(dt)
        s["bias"] = (0.1 * _normal(gen, w)).to(dt)
        s["x"] += 0.5
        if step and case["residual"]:
            s["grad_total"] = (_normal(gen, n, w) * 0.01).to(dt)
    else:
        # the generator's state, as a training program keeps it: seed and number of the step
        s["seed"] = torch.randint(0, 2 ** 40, (2,), generator=gen, device=DEV)
        s["layer"] = 3
    if step:
        s["grad"] = (_normal(gen, n, w) * 0.01).to(dt)
        for name in ("x", "residual", "weight", "bias"):
            if s.get(name) is not None:
                s[name].requires_grad_()
    return s


# ---------------------------------------------------------------------------- one pass
def _plain_embed(s):
    ids = s["ids"].long()
    if s["offsets"] is None:
        ids, first, last = ids[:, None], 0, s["entries"]
    else:
        first, last = s["offsets"][:-1], s["offsets"][1:]
    at = ids + first
    there = (ids >= 0) & (at < last)
    at = torch.where(there, at, 0)
    if s["way"] == "lookup":
        rows = s["table"][at.reshape(-1)].float().view(*at.shape, -1)
        return ((rows * there[:, :, None]).sum(1) * s["scale"]).to(s["table"].dtype)
    n, k = at.shape
    grad = s["grad"].float()[:, None, :].expand(-1, k, -1) * there[:, :, None]
    out = torch.zeros(s["entries"], s["width"], device=DEV)
    out.index_add_(0, at.reshape(-1), grad.reshape(n * k, -1))
    return (out * s["scale"]).to(s["grad"].dtype)


def _plain_layer_norm(s):
    dt = s["x"].dtype
    with torch.no_grad():
        t, total = s["x"].float(), None
        if s["residual"] is not None:
            total = (t + s["residual"].float()).to(dt)  # the norm is the rounded sum's
            t = total.float()
        w, b = s["weight"].float(), s["bias"].float()
        c = t - t.mean(1, keepdim=True)
        r = 1 / torch.sqrt((c * c).mean(1, keepdim=True) + EPS)
        h = c * r
        y = (h * w + b).to(dt)
        if s["way"] == "forward":
            return y, total
        g = s["grad"].float()
        a = g * w
        dx = r * (a - a.mean(1, keepdim=True) - h * (a * h).mean(1, keepdim=True))
        dw, db = (g * h).sum(0).to(dt), g.sum(0).to(dt)
        if total is None:
            return y, dx.to(dt), dw, db
        dx = (dx + s["grad_total"].float()).to(dt)
        return y, total, dx, dx, dw, db


def _words(c0, c1, c2, c3, k0, k1):
    """Philox4x32-10 (Salmon, Moraes, Dror, Shaw 2011) on 32-bit words held in int64."""
    low = 0xFFFFFFFF
    for _ in range(10):
        a, b = c0 * 0xD2511F53, c2 * 0xCD9E8D57
        c0, c1, c2, c3 = ((b >> 32) & low) ^ c1 ^ k0, b & low, ((a >> 32) & low) ^ c3 ^ k1, a & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return c0, c1, c2, c3


def _plain_keep(s):
    """Which elements stay: 32 random bits against p, the upper 16 of them from one block of words
    for each 8 neighbours of a row, the lower 16 from another."""
    n, w = s["x"].shape
    seed, step = s["seed"][0], s["seed"][1]
    unit = torch.arange((w + 7) // 8, device=DEV).expand(n, -1)
    row = torch.arange(n, device=DEV)[:, None].expand_as(unit)
    parts = []
    for low in (0, 1):
        words = _words(unit, row, (step & 0xFFFFFFFF).expand_as(unit),
                       torch.full_like(unit, 2 * s["layer"] + low), seed & 0xFFFFFFFF,
                       (seed >> 32) & 0xFFFFFFFF)
        halves = torch.stack([h for v in words for h in (v & 0xFFFF, v >> 16)], 2)
        parts.append(halves.reshape(n, -1)[:, :w])
    return (parts[0] << 16 | parts[1]) >= round(s["p"] * 2 ** 32)


def _plain_dropout(s):
    dt = s["x"].dtype
    with torch.no_grad():
        keep = _plain_keep(s)
        out = torch.where(keep, s["x"].float() * (1 / (1 - s["p"])), 0.0)
        if s["residual"] is not None:
            out = out + s["residual"].float()
        if s["way"] == "forward":
            return out.to(dt)
        dx = torch.where(keep, s["grad"].float() * (1 / (1 - s["p"])), 0.0).to(dt)
        return (out.to(dt), dx) + ((s["grad"],) if s["residual"] is not None else ())


def _column(v):
    return v.double()[:, None] if torch.is_tensor(v) else v


def _plain_sample(s):
    n, c = s["logits"].shape
    z, order = torch.sort(s["logits"].float() + 0.0, dim=1, descending=True, stable=True)
    z = z.double()
    top = z[:, :1]
    T, top_k, top_p, min_p = (_column(s[name]) for name in ("temperature", "top_k", "top_p", "min_p"))
    rank = torch.arange(c, device=DEV)[None]
    stays = ((rank < top_k) | (torch.as_tensor(top_k, device=DEV) <= 0)) & (z > -math.inf)
    mass = torch.where(stays, torch.exp((z - top) / T), 0.0)
    before = torch.cumsum(mass, 1) - mass
    if torch.is_tensor(top_p) or top_p < 1:
        limit = torch.where(torch.as_tensor(top_p, device=DEV) < 1,
                            top_p * mass.sum(1, keepdim=True), math.inf)
        stays &= (before < limit) | (rank == 0)
    floor = torch.log(min_p) if torch.is_tensor(min_p) else \
        (math.log(min_p) if min_p > 0 else -math.inf)
    stays &= z >= top + T * floor
    mass = torch.where(stays, mass, 0.0)
    # the draw runs over the classes in their own order
    mass = torch.zeros_like(mass).scatter_(1, order, mass)
    sums = torch.cumsum(mass, 1)
    u = s["u"].double()[:, None]
    at = (sums <= u * sums[:, -1:]).sum(1, keepdim=True).clamp_(max=c - 1)
    return at[:, 0].to(torch.int32), torch.log(mass.gather(1, at) / sums[:, -1:])[:, 0].float()


def _own(s):
    import paper_2405_12491_amd as B
    step = s.get("way") == "step"
    if s["op"] == "embed" and s["way"] == "lookup":
        return B.embed(s["ids"], s["table"], scale=s["scale"], offsets=s["offsets"])
    if s["op"] == "embed":
        return B.embed_grad(s["ids"], s["grad"], s["entries"], scale=s["scale"],
                            offsets=s["offsets"])
    if s["op"] == "layer_norm":
        y, total = B.layer_norm(s["x"], s["weight"], s["bias"], residual=s["residual"], eps=EPS)
        if not step:
            return y, total
        if total is None:
            return (y.detach(),) + torch.autograd.grad(y, (s["x"], s["weight"], s["bias"]), s["grad"])
        grads = torch.autograd.grad((y, total), (s["x"], s["residual"], s["weight"], s["bias"]),
                                    (s["grad"], s["grad_total"]))
        return (y.detach(), total.detach()) + grads
    if s["op"] == "dropout":
        out = B.dropout(s["x"], s["p"], s["seed"], residual=s["residual"], layer=s["layer"])
        if not step:
            return out
        leaves = (s["x"],) if s["residual"] is None else (s["x"], s["residual"])
        return (out.detach(),) + torch.autograd.grad(out, leaves, s["grad"])
    return B.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"],
                    top_p=s["top_p"], min_p=s["min_p"])


def run(state):
    if own:
        return _own(state)
    return {"embed": _plain_embed, "layer_norm": _plain_layer_norm, "dropout": _plain_dropout,
            "sample": _plain_sample}[state["op"]](state)


def work(case):
    n, w, e = case["rows"], case["width"], BYTES[case["dtype"]]
    if case["op"] == "embed":
        pairs, entries = n * case["slots"], case["entries"]
        table = (min(pairs, entries) if case["way"] == "lookup" else entries) * w * e
        return {"bytes": 4 * pairs + table + n * w * e, "flops": pairs * w}
    if case["op"] == "layer_norm":
        rows = 4 if case["residual"] else 2
        if case["way"] == "step":  # gradient and norm's rows in, the rows' gradient out
            rows += 4 if case["residual"] else 3
        return {"bytes": n * w * e * rows, "flops": n * w * (24 if case["way"] == "step" else 8)}
    if case["op"] == "dropout":
        rows = (3 if case["residual"] else 2) + (2 if case["way"] == "step" else 0)
        return {"bytes": n * w * e * rows, "flops": 12 * n * w}
    return {"bytes": n * w * e + 12 * n, "flops": 4 * n * w}


# ------------------------------------------------------------------- the definition, 64 bits
def _exact_embed(s):
    n, k = s["rows"], s["slots"]
    out = torch.zeros(n if s["way"] == "lookup" else s["entries"], s["width"], dtype=torch.float64,
                      device=DEV)
    ids = s["ids"].view(n, k).long()
    begin = [0, s["entries"]] if s["offsets"] is None else s["offsets"].tolist()
    for t in range(k):
        row = torch.nonzero((ids[:, t] >= 0) & (ids[:, t] < begin[t + 1] - begin[t]))[:, 0]
        entry = ids[row, t] + begin[t]
        if s["way"] == "lookup":
            out[row] += s["table"][entry].double()
        else:
            out.index_add_(0, entry, s["grad"][row].double())
    return out.mul_(s["scale"])


def _exact_layer_norm(s):
    x, total = s["x"].detach(), None
    if s["residual"] is not None:
        total = x.double() + s["residual"].detach().double()
        x = total.to(x.dtype)
    x, w, b = x.double(), s["weight"].detach().double(), s["bias"].detach().double()
    var, mean = torch.var_mean(x, dim=1, correction=0, keepdim=True)
    std = (var + EPS).sqrt()
    h = x.sub_(mean).div_(std)
    y = torch.addcmul(b, h, w)
    if s["way"] == "forward":
        return y, total
    g = s["grad"].double()
    dw, db = torch.mul(g, h).sum(0), g.sum(0)
    g.mul_(w)
    along = torch.linalg.vecdot(g, h, dim=1)[:, None] / s["width"]
    dx = g.sub_(g.mean(1, keepdim=True)).sub_(h.mul_(along)).div_(std)
    if total is None:
        return y, dx, dw, db
    dx += s["grad_total"].double()
    return y, total, dx, dx, dw, db


def _exact_bits(s, tail, row0, rows):
    """16 random bits of each of `rows` rows' elements: the generator on words of two 16-bit digits."""
    def times(x, m):  # the upper and the lower word of a product
        lo, mid0, mid1 = (x & 65535) * (m & 65535), (x >> 16) * (m & 65535), (x & 65535) * (m >> 16)
        mid = (lo >> 16) + (mid0 & 65535) + (mid1 & 65535)
        return ((x >> 16) * (m >> 16) + (mid0 >> 16) + (mid1 >> 16) + (mid >> 16),
                (mid & 65535) << 16 | lo & 65535)

    seed, step = (int(v) for v in s["seed"].tolist())
    units = (s["width"] + 7) // 8
    ctr = torch.empty(4, rows, units, dtype=torch.int64, device=DEV)
    ctr[0] = torch.arange(units, device=DEV)
    ctr[1] = torch.arange(row0, row0 + rows, device=DEV)[:, None]
    ctr[2], ctr[3] = step % 2 ** 32, tail
    for r in range(10):
        key = (seed + r * 0x9E3779B9) % 2 ** 32, ((seed >> 32) + r * 0xBB67AE85) % 2 ** 32
        hi0, lo0 = times(ctr[0], 0xD2511F53)
        hi1, lo1 = times(ctr[2], 0xCD9E8D57)
        ctr = torch.stack([hi1 ^ ctr[1] ^ key[0], lo1, hi0 ^ ctr[3] ^ key[1], lo0])
    halves = torch.stack([ctr % 65536, ctr // 65536], 1).flatten(0, 1)
    return halves.permute(1, 2, 0).reshape(rows, units * 8)[:, :s["width"]]


def _exact_dropout(s):
    n, most = s["rows"], max(1, 4_000_000 // s["width"])
    up = 1 / (1 - s["p"])
    out, dx = [], []
    for row0 in range(0, n, most):
        rows = min(most, n - row0)
        part = slice(row0, row0 + rows)
        drawn = (_exact_bits(s, 2 * s["layer"], row0, rows) * 65536
                 + _exact_bits(s, 2 * s["layer"] + 1, row0, rows))
        factor = (drawn >= round(s["p"] * 2 ** 32)).double() * up
        v = s["x"].detach()[part].double() * factor
        if s["residual"] is not None:
            v += s["residual"].detach()[part].double()
        out.append(v)
        if s["way"] == "step":
            dx.append(s["grad"][part].double() * factor)
    if s["way"] == "forward":
        return torch.cat(out)
    same = (s["grad"].double(),) if s["residual"] is not None else ()
    return (torch.cat(out), torch.cat(dx)) + same


def _exact_sample(s):
    n, c = s["logits"].shape
    logp = torch.empty(n, dtype=torch.float64, device=DEV)

    def of(name, r):
        return float(s[name][r]) if torch.is_tensor(s[name]) else float(s[name])

    draws = s["u"].tolist()
    for r in range(n):
        z = s["logits"][r].double()
        k = int(of("top_k", r))
        k = c if k <= 0 else min(k, c)
        T, p, least = of("temperature", r), of("top_p", r), of("min_p", r)
        value, cls = torch.sort(z + 0.0, descending=True, stable=True)
        value, cls = value[:k], cls[:k]
        share = torch.softmax(value / T, 0)
        m = k
        if p < 1:
            m = max(1, min(m, int(torch.searchsorted(torch.cumsum(share, 0), p)) + 1))
        if least > 0:
            m = min(m, int((value >= value[0] + T * math.log(least)).sum()))
        cls, by = torch.sort(cls[:m])
        share = torch.softmax(value[:m] / T, 0)[by]
        chosen = int(torch.searchsorted(torch.cumsum(share, 0), draws[r], right=True))
        logp[r] = torch.log(share[min(chosen, m - 1)])
    return None, logp


def exact(case, seed):
    if case["op"] == "sample" and case["rows"] > 4_000:
        return None  # row by row it takes longer than is useful
    return {"embed": _exact_embed, "layer_norm": _exact_layer_norm, "dropout": _exact_dropout,
            "sample": _exact_sample}[case["op"]](prepare(case, seed))
