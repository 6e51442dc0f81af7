"""Workloads of the operators around a cache held in 8 or 4 bits and of the log
probabilities that a server answers with, for timing and for comparing outputs.

  attend    Pages.plan, then ldr.attend of every layer over a cache of coded rows:
            the open rows of each sequence attend to all its rows
  write     the rows of a pass go into such a cache (room, codes) and come back
            as the values that they now stand for
  read      ranges of rows of such a cache as bf16 rows
  logprobs  ldr.logprobs: log probability and rank of a given token of each row
            of logits, the row's entropy, its top alternatives

With `own` false the same results come from elementary torch operations on the
same inputs; with `own` true from the library. Head layouts and vocabularies are
those of the library's shapes (the Qwen3-8B and Qwen3-32B drafters, the small bf16
model, the layout of the Tiny model).

Codes: 32 consecutive dimensions of a row share a scale 2^e, the smallest with
max |x| <= 7 * 2^e (4 bits, e2m1) or 464 * 2^e (8 bits, e4m3); x / 2^e is rounded
to the nearest code, ties to the even one.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
F64 = torch.float64
BF = torch.bfloat16

# query heads, K/V heads, head dim of the shapes
HEADS = {"8b": (32, 8, 128), "32b": (64, 8, 128), "mini": (8, 2, 128), "tiny": (4, 4, 64)}
# bits: what a scale's limit is, largest code, lowest exponent, largest value coded
CODES = {4: (7.0, 6.0, -125, 1.5 * 2.0 ** 127), 8: (464.0, 448.0, -117, 1.875 * 2.0 ** 127)}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# --------------------------------------------------------------------- cases

def _attend(name, bits, heads, batch, new, shared, rows, layers, page=64):
    return {"name": name, "kind": "attend", "bits": bits, "heads": heads, "batch": batch,
            "new": new, "shared": shared, "rows": rows, "layers": layers, "page": page}


def _rows(name, op, bits, batch, new, rows, layers, heads="8b", page=64):
    return {"name": name, "kind": op, "bits": bits, "heads": heads, "batch": batch, "new": new,
            "rows": rows, "layers": layers, "page": page}


def _logprobs(name, batch, rows, vocab, top, temperature=1.0, ragged=False):
    return {"name": name, "kind": "logprobs", "batch": batch, "rows": rows, "vocab": vocab,
            "top": top, "temperature": temperature, "ragged": ragged}


def listed():
    return [
        # the smallest call: a decoded token of one request of the small layout
        _attend("attend4-tiny-b1", 4, "tiny", 1, 1, 0, 1000, 1, 32),
        # one decoded token of each of 16 unrelated requests
        _attend("attend4-decode-b16", 4, "8b", 16, 1, 0, 16384, 5),
        # the target's pass over the drafted blocks of 16 unrelated requests
        _attend("attend4-verify-b16", 4, "8b", 16, 17, 0, 8192, 5),
        # one long document in an interactive session, its drafted block
        _attend("attend8-long-b1", 8, "8b", 1, 17, 0, 65536, 2),
        # one decoded token of each of 64 samples of one long prompt
        _attend("attend8-decode-b64", 8, "8b", 64, 1, 32768, 300, 2),
        # prefill: the next chunk of two requests behind a common system prompt
        _attend("attend4-prefill-b2", 4, "8b", 2, 512, 4096, 4096, 2),
        # the rows of one verification pass of a serving batch
        _rows("write4-b16", "write", 4, 16, 17, 4096, 5),
        # two prompts as they are prefilled
        _rows("write8-b2", "write", 8, 2, 2048, 2048, 5),
        # the prefixes of a batch, to build the drafter's views from
        _rows("read4-b16", "read", 4, 16, 4096, 4200, 5),
        # one interactive request: the token just decoded and five alternatives
        _logprobs("logprobs-b1", 1, 1, 151936, 5),
        # a verified batch: the tokens emitted by sequences that stopped at different places
        _logprobs("logprobs-b16", 16, 17, 151936, 20, 0.7, True),
        # a prompt is scored
        _logprobs("logprobs-prompt", 1, 1024, 151936, 1),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choices(("attend", "write", "read", "logprobs"), (8, 3, 3, 5))[0]
    bits = rng.choice((4, 4, 8))
    page = rng.choice((32, 64, 64, 128, 256))
    if kind == "logprobs":
        vocab = rng.choice((151936, 151936, 128257, 32000, 5003, 4099))
        batch = _log_int(rng, 1, 64)
        return {"kind": kind, "batch": batch, "rows": _log_int(rng, 1, 1024 // batch),
                "vocab": vocab, "top": rng.choice((0, 1, 5, 20, rng.randint(2, 64))),
                "temperature": rng.choice((1.0, 0.7, 1.3)), "ragged": rng.random() < 0.5}
    if kind == "attend":
        heads = rng.choices(("8b", "32b", "mini", "tiny"), (6, 2, 3, 2))[0]
        hq, hkv, d = HEADS[heads]
        new = rng.choice((1, 1, 17, rng.randint(2, 16), _log_int(rng, 18, 512)))
        batch = _log_int(rng, 1, 64)
        shared = rng.choice((0, _log_int(rng, 32, 32768), _log_int(rng, 32, 32768)))
        rows = new + _log_int(rng, 1, 16384)
        layers = rng.randint(1, 5)
        # no more work than the largest listed case, and caches of at most 2^18 rows
        top = work(_attend("", 8, "8b", 64, 1, 32768, 300, 2))["flops"]
        while batch > 1 and (batch * rows + shared > 1 << 18 or
                             4.0 * layers * batch * new * hq * d * (shared + rows) > top):
            batch = (batch + 1) // 2
        while layers > 1 and 4.0 * layers * batch * new * hq * d * (shared + rows) > top:
            layers -= 1
        while rows > new + 1 and 4.0 * batch * new * hq * d * (shared + rows) > top:
            rows, shared = new + (rows - new) // 2, shared // 2
        return {"kind": kind, "bits": bits, "heads": heads, "batch": batch, "new": new,
                "shared": shared, "rows": rows, "layers": layers, "page": page}
    heads = rng.choice(("8b", "8b", "32b", "mini", "tiny"))
    batch = _log_int(rng, 1, 64)
    layers = rng.randint(1, 5)
    if kind == "write":
        new = rng.choice((1, 17, rng.randint(2, 16), _log_int(rng, 18, max(18, 4096 // batch))))
        rows = _log_int(rng, 1, max(1, 65536 // batch))
    else:
        new = _log_int(rng, 1, 65536 // batch)
        rows = new + rng.randint(0, 300)
    return {"kind": kind, "bits": bits, "heads": heads, "batch": batch, "new": new, "rows": rows,
            "layers": layers, "page": page}


# -------------------------------------------------------------------- inputs

def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(int(seed))
    return g


def _randn(g, shape, dtype=torch.float32):
    return torch.randn(shape, generator=g, device=DEV, dtype=dtype)


def _kv_rows(g, shape):
    """bf16 rows as projections leave them: some dimensions larger than the others."""
    wide = torch.exp(0.7 * _randn(g, shape[-1:]))
    return (_randn(g, shape) * wide).to(BF)


def _quantise(x, bits):
    """Rows [..., d] -> the codes' values as whole numbers of their grid (fp32)
    and the exponents [..., d / 32]; a block that is not finite has exponent 128."""
    limit, most, low, top = CODES[bits]
    x = x.float()
    bad = (~torch.isfinite(x)).unflatten(-1, (-1, 32)).any(-1)
    x = x.nan_to_num(0.0, top, -top).clamp(-top, top).unflatten(-1, (-1, 32))
    f, e = torch.frexp(x.abs().amax(-1))
    fl, el = math.frexp(limit)
    e = (e.int() - el + (f > fl)).clamp(min=low)
    # in two steps: 2^-e alone may be no fp32 number
    half = torch.div(e, 2, rounding_mode="floor")
    y = torch.ldexp(torch.ldexp(x, -half[..., None]), (half - e)[..., None])
    a = y.abs()
    p = torch.frexp(a)[1].int() - 1                     # floor(log2 a)
    step = torch.ldexp(torch.ones_like(a), p.clamp(min=0 if bits == 4 else -6) - (1 if bits == 4 else 3))
    q = torch.copysign((torch.round(a / step) * step).clamp(max=most), y)
    return q.flatten(-2), torch.where(bad, 128, e)


def _to_codes(q, bits):
    """Values of the grid [..., d] -> codes: 4 bits two a byte, the even dimension low."""
    if bits == 8:
        return q.to(torch.float8_e4m3fn).view(torch.uint8)
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], device=q.device)
    c = torch.bucketize(q.abs(), edges).to(torch.uint8) | (torch.signbit(q).to(torch.uint8) << 3)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _to_values(c, e, bits):
    """Codes [..., d / 2 or d] and exponent bytes [..., d / 32] -> fp32 values."""
    if bits == 8:
        q = c.view(torch.float8_e4m3fn).float()
    else:
        t = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=c.device)
        q = t[torch.stack((c & 15, c >> 4), -1).flatten(-2).int()]
    s = torch.where(e == 255, math.nan, torch.ldexp(torch.ones((), device=c.device), e.int() - 127))
    return (q.unflatten(-1, (-1, 32)) * s[..., None]).flatten(-2)


def _lengths(case):
    """Rows of each sequence's own (all its rows, the open ones at their end)
    and its open rows: a part of the batch has fewer, as requests do."""
    b, new, rows = case["batch"], case["new"], case["rows"]
    opened = [new if new < 4 else new - i % 3 for i in range(b)]
    return [max(o, rows - (i * 37) % (rows // 4 + 1)) for i, o in enumerate(opened)], opened


class _State:
    """A cache of plain tensors: codes and exponents by rows, bookkeeping in one
    int32 buffer."""

    def __init__(self, case, n_pages, max_pages):
        hq, self.hkv, self.d = HEADS[case["heads"]]
        L, self.bits, batch = case["layers"], case["bits"], case["batch"]
        self.page, self.n_pages, self.batch, self.max_pages = case["page"], n_pages, batch, max_pages
        shape = (L, 2, n_pages, self.hkv, self.page)
        self.codes = torch.zeros(*shape, self.d * self.bits // 8, dtype=torch.uint8, device=DEV)
        self.scales = torch.zeros(*shape, self.d // 32, dtype=torch.uint8, device=DEV)
        self.state = torch.zeros(2 * batch + batch * max_pages + n_pages, dtype=torch.int32,
                                 device=DEV)
        self.rows, self.open, t, self.refs = self.state.split(
            [batch, batch, batch * max_pages, n_pages])
        self.table = t.view(batch, max_pages)

    def put(self, layer, which, q, e):
        self.codes[layer, which] = _to_codes(q, self.bits)
        self.scales[layer, which] = (e + 127).to(torch.uint8)

    def values(self, layer, which, ids):
        """fp32 rows [ids][hkv][page][d] of pages."""
        return _to_values(self.codes[layer, which][ids], self.scales[layer, which][ids], self.bits)


def _put(p, bits, layer, which, q, e):
    """The same codes in the library's pool: K codes by rows, V codes by pairs of
    dimensions; behind them the scales, K's by rows, V's by blocks."""
    n = q.shape[0]
    c = _to_codes(q, bits)                                   # [pages][hkv][page][bytes]
    s = (e + 127).to(torch.uint8)                            # [pages][hkv][page][d / 32]
    if which == 1:                                           # a pair is one byte or two
        c = c.unflatten(-1, (-1, bits // 4)).transpose(2, 3).flatten(3)
        s = s.transpose(2, 3)
    p.pool[layer, which] = torch.cat((c.reshape(n, p.hkv, -1), s.reshape(n, p.hkv, -1)), -1)


def _cache(case, g, n_pages, max_pages, table, rows, opened):
    """A running cache: page ids per sequence, rows, open rows, as many references
    on a page as tables hold it, and rows in all its pages."""
    if own:
        from paper_2609_37029_amd import ldr
        hq, hkv, d = HEADS[case["heads"]]
        p = ldr.Pages(case["layers"], hkv, d, case["page"], n_pages, case["batch"], max_pages,
                      codes="mxfp%d" % case["bits"]).init()
    else:
        p = _State(case, n_pages, max_pages)
    p.rows.copy_(torch.tensor(rows, dtype=torch.int32))
    p.open.copy_(torch.tensor(opened, dtype=torch.int32))
    t = torch.full((p.batch, max_pages), -1, dtype=torch.int32)
    for b, ids in enumerate(table):
        t[b, :len(ids)] = torch.tensor(ids, dtype=torch.int32)
    p.table.copy_(t)
    p.refs.copy_(torch.bincount(t[t >= 0].long(), minlength=n_pages).int())
    for layer in range(case["layers"]):
        for which in (0, 1):
            q, e = _quantise(_kv_rows(g, (n_pages, p.hkv, case["page"], p.d)), case["bits"])
            if own:
                _put(p, case["bits"], layer, which, q, e)
            else:
                p.put(layer, which, q, e)
    return p


def _prepare_attend(case, seed):
    g = _gen(seed)
    hq, hkv, d = HEADS[case["heads"]]
    page, b, L = case["page"], case["batch"], case["layers"]
    own_rows, opened = _lengths(case)
    head = case["shared"] // page                 # pages of the common prefix
    tails = [-(-r // page) for r in own_rows]
    used = head + sum(tails)
    n_pages = used + used // 16 + 1
    ids = torch.randperm(n_pages, generator=torch.Generator().manual_seed(int(seed))).tolist()
    table, at = [], head
    for n in tails:
        table.append(ids[:head] + ids[at:at + n])
        at += n
    p = _cache(case, g, n_pages, max(len(t) for t in table) + 2, table,
               [head * page + r for r in own_rows], opened)
    st = {"case": case, "pages": p, "cols": max(len(t) for t in table),
          "q": _randn(g, (L, b, case["new"], hq, d)).to(BF),
          "o": torch.zeros(L, b, case["new"], hq, d, dtype=BF, device=DEV),
          "lse": torch.zeros(L, b, case["new"], hq, device=DEV)}
    if own:
        st["ws"] = torch.empty(p.attend_workspace_bytes(hq, case["new"]), dtype=torch.uint8,
                               device=DEV)
    return st


def _prepare_rows(case, seed):
    g = _gen(seed)
    rng = np.random.default_rng(int(seed))
    hq, hkv, d = HEADS[case["heads"]]
    page, b, new = case["page"], case["batch"], case["new"]
    n = rng.integers((new + 1) // 2, new + 1, b)
    rows = [max(int(k) if case["kind"] == "read" else 1,
                case["rows"] - (i * 37) % (case["rows"] // 4 + 1)) for i, k in enumerate(n)]
    need = [-(-r // page) for r in rows]
    n_pages = sum(need) + (b * (-(-new // page) + 1) if case["kind"] == "write" else 1)
    ids = rng.permutation(n_pages).tolist()
    table, at = [], 0
    for k in need:
        table.append(ids[at:at + k])
        at += k
    p = _cache(case, g, n_pages, max(need) + -(-new // page) + 1, table, rows, [0] * b)
    shape = (b, new, case["layers"], hkv, d)
    st = {"case": case, "pages": p, "before": p.state.clone(),
          "n": torch.tensor(n, dtype=torch.int32, device=DEV),
          "back": tuple(torch.zeros(shape, dtype=BF, device=DEV) for _ in range(2))}
    if case["kind"] == "write":
        st.update(K=_kv_rows(g, shape), V=_kv_rows(g, shape), first=p.rows.clone())
    else:
        first = [int(rng.integers(0, r - k + 1)) for r, k in zip(rows, n)]
        st["first"] = torch.tensor(first, dtype=torch.int32, device=DEV)
    return st


def _prepare_logprobs(case, seed):
    """Logits with a few likely tokens a row; the given token is mostly one of them."""
    g = _gen(seed)
    b, R, V = case["batch"], case["rows"], case["vocab"]
    z = _randn(g, (b, R, V)).mul_(2.0)
    likely = torch.randint(0, V, (b, R, 8), generator=g, device=DEV)
    z.scatter_add_(2, likely, 8.0 + 3.0 * _randn(g, (b, R, 8)))
    y = likely[..., 0]
    other = torch.randint(0, V, (b, R), generator=g, device=DEV)
    y = torch.where(torch.rand(b, R, generator=g, device=DEV) < 0.8, y, other).to(torch.int32)
    n = None
    if case["ragged"]:
        n = torch.randint(1, R + 1, (b,), generator=g, device=DEV).to(torch.int32)
    k = case["top"]
    out = (torch.zeros(b, R, device=DEV), torch.zeros(b, R, device=DEV),
           torch.zeros(b, R, dtype=torch.int32, device=DEV),
           torch.zeros(b, R, k, dtype=torch.int32, device=DEV), torch.zeros(b, R, k, device=DEV))
    st = {"case": case, "z": z, "y": y, "n": n, "out": out}
    if own:
        from paper_2609_37029_amd import ldr
        st["ws"] = torch.empty(ldr.logprobs_workspace_bytes(b, R, V, k), dtype=torch.uint8,
                               device=DEV)
    return st


def prepare(case, seed):
    return {"attend": _prepare_attend, "write": _prepare_rows, "read": _prepare_rows,
            "logprobs": _prepare_logprobs}[case["kind"]](case, seed)


# --------------------------------------------------------------- plain forms

def _attend_plain(st):
    """softmax(q k^T / sqrt(d)) v of every sequence over its decoded pages."""
    case, p, cols = st["case"], st["pages"], st["cols"]
    hq, hkv, d = HEADS[case["heads"]]
    b, S, page = case["batch"], case["new"], case["page"]
    n = cols * page
    key = torch.arange(n, device=DEV)
    i = torch.arange(S, device=DEV)
    step = max(1, (1 << 30) // (n * hkv * (d + S * (hq // hkv))))   # sequences a part
    for layer in range(case["layers"]):
        for lo in range(0, b, step):
            hi = min(b, lo + step)
            ids = p.table[lo:hi, :cols].clamp(min=0).long()
            k = p.values(layer, 0, ids).transpose(1, 2).reshape(hi - lo, hkv, n, d)
            v = p.values(layer, 1, ids).transpose(1, 2).reshape(hi - lo, hkv, n, d)
            q = st["q"][layer, lo:hi].float().view(hi - lo, S, hkv, hq // hkv, d)
            q = q.permute(0, 2, 3, 1, 4).reshape(hi - lo, hkv, -1, d)
            s = (q @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
            s = s.view(hi - lo, hkv, hq // hkv, S, n)
            # row i of the open rows sees the keys up to its own position
            last = (p.rows - p.open)[lo:hi, None] + i
            seen = (key <= last[..., None]) & (i < p.open[lo:hi, None])[..., None]
            s = s.masked_fill_(~seen[:, None, None], -math.inf)
            m = s.amax(-1, keepdim=True)
            e = s.sub_(torch.where(m == -math.inf, 0.0, m)).exp_()
            total = e.sum(-1)
            o = e.view(hi - lo, hkv, -1, n) @ v
            o = o.view(hi - lo, hkv, hq // hkv, S, d) / total.clamp(min=1e-30)[..., None]
            lse = m[..., 0] + total.log()
            here = (i < p.open[lo:hi, None])[..., None]       # the other rows stay as they are
            o = o.permute(0, 3, 1, 2, 4).reshape(hi - lo, S, hq, d).to(BF)
            lse = lse.permute(0, 3, 1, 2).reshape(hi - lo, S, hq)
            st["o"][layer, lo:hi] = torch.where(here[..., None], o, st["o"][layer, lo:hi])
            st["lse"][layer, lo:hi] = torch.where(here, lse, st["lse"][layer, lo:hi])
    return {"o": st["o"], "lse": st["lse"]}


def _reserve_plain(p, n, new):
    """Room for n more rows of each sequence: the lowest free pages, in the order
    of the sequences (no page is shared here)."""
    page = p.page
    first = (p.rows.long() + page - 1) // page
    need = (p.rows + n + page - 1) // page - first
    start = need.cumsum(0) - need
    free = torch.argsort((p.refs > 0).int(), stable=True)
    for t in range(-(-new // page) + 1):
        at = (first + t).clamp(max=p.max_pages - 1)[:, None]
        got = free[(start + t).clamp(max=p.n_pages - 1)].int()[:, None]
        p.table.scatter_(1, at, torch.where((t < need)[:, None], got, p.table.gather(1, at)))
    p.rows.add_(n)
    p.open.copy_(n)
    t = p.table.reshape(-1).long()
    p.refs.zero_().scatter_add_(0, t.clamp(min=0), (t >= 0).int())


def _places(p, first, n, new):
    """Page and row in it of rows first .. first + n of each sequence; rows behind
    them are the last one again."""
    r = torch.minimum(torch.arange(new, device=DEV), n[:, None] - 1)
    pos = first[:, None].long() + r
    return p.table.gather(1, pos // p.page).clamp(min=0).long(), pos % p.page, r.long()


def _write_plain(p, n, K, V):
    pg, off, r = _places(p, p.rows - n, n, K.shape[1])
    for which, x in ((0, K), (1, V)):
        x = x.take_along_dim(r[..., None, None, None], 1)
        q, e = _quantise(x, p.bits)
        c, e = _to_codes(q, p.bits), (e + 127).to(torch.uint8)
        for layer in range(K.shape[2]):
            p.codes[layer, which][pg, :, off] = c[:, :, layer]
            p.scales[layer, which][pg, :, off] = e[:, :, layer]


def _read_plain(p, first, n, back):
    new = back[0].shape[1]
    pg, off, r = _places(p, first, n, new)
    here = (torch.arange(new, device=DEV) < n[:, None])[..., None, None]
    for which, out in enumerate(back):
        for layer in range(out.shape[2]):
            x = _to_values(p.codes[layer, which][pg, :, off], p.scales[layer, which][pg, :, off],
                           p.bits).to(BF)
            out[:, :, layer] = torch.where(here, x, out[:, :, layer])


def _logprobs_plain(st):
    case, z, y = st["case"], st["z"], st["y"].long()
    x = z if case["temperature"] == 1.0 else z / case["temperature"]
    x = x - x.amax(-1, keepdim=True)
    e = x.exp()
    s = e.sum(-1)
    ls = s.log()
    xy = x.gather(2, y[..., None])
    zy = z.gather(2, y[..., None])
    before = torch.arange(case["vocab"], device=DEV) < y[..., None]
    rank = ((z > zy) | ((z == zy) & before)).sum(-1)
    order = torch.sort(z, stable=True, dim=-1, descending=True)[1][..., :case["top"]]
    new = (xy[..., 0] - ls, ls - (e * x).sum(-1) / s, rank.int(), order.int(),
           x.gather(2, order) - ls[..., None])
    if st["n"] is not None:                    # the other rows stay as they are
        here = torch.arange(case["rows"], device=DEV) < st["n"][:, None]
        new = tuple(torch.where(here if a.dim() == 2 else here[..., None], a, b)
                    for a, b in zip(new, st["out"]))
    return new


# ----------------------------------------------------------------------- run

def run(st):
    case = st["case"]
    kind = case["kind"]
    p = st.get("pages")
    if kind == "write":
        p.state.copy_(st["before"])     # the cache as it was before this pass
    if not own:
        if kind == "attend":
            return _attend_plain(st)
        if kind == "logprobs":
            return _logprobs_plain(st)
        if kind == "write":
            _reserve_plain(p, st["n"], case["new"])
            _write_plain(p, st["n"], st["K"], st["V"])
        _read_plain(p, st["first"], st["n"], st["back"])
    else:
        from paper_2609_37029_amd import ldr
        if kind == "attend":
            plan = p.plan(HEADS[case["heads"]][0], case["new"], workspace=st["ws"])
            for layer in range(case["layers"]):
                ldr.attend(plan, layer, st["q"][layer], out=st["o"][layer], lse=st["lse"][layer])
            return {"o": st["o"], "lse": st["lse"]}
        if kind == "logprobs":
            return ldr.logprobs(st["z"], st["y"], top_n=case["top"],
                                temperature=case["temperature"], n_rows=st["n"], out=st["out"],
                                workspace=st["ws"])
        if kind == "write":
            p.reserve(st["n"], case["new"])
            p.write(st["K"], st["V"])
        p.read(st["first"], st["n"], out=st["back"])
    if kind == "read":
        return {"K": st["back"][0], "V": st["back"][1]}
    return {"K": st["back"][0], "V": st["back"][1], "rows": p.rows, "open": p.open,
            "table": p.table, "refs": p.refs}


# ---------------------------------------------------------------------- work

def work(case):
    kind = case["kind"]
    if kind == "logprobs":
        b, R, V = case["batch"], case["rows"], case["vocab"]
        rows = b * R if not case["ragged"] else b * (R + 1) / 2
        return {"bytes": rows * (4.0 * V + 16 + 8 * case["top"]), "flops": 4.0 * rows * V}
    hq, hkv, d = HEADS[case["heads"]]
    b, L = case["batch"], case["layers"]
    row = 2.0 * hkv * d * L * (case["bits"] / 8 + 1 / 32)   # K and V of one row in all layers
    if kind == "attend":
        rows, opened = _lengths(case)
        head = case["shared"] // case["page"] * case["page"]
        pairs = sum(sum(head + r - o + i + 1 for i in range(o)) for r, o in zip(rows, opened))
        return {"bytes": row * (head + sum(rows)) + L * sum(opened) * hq * (4.0 * d + 4.0),
                "flops": 4.0 * L * hq * d * pairs}
    n = b * ((case["new"] + 1) // 2 + case["new"]) / 2
    plain = 4.0 * hkv * d * L                               # the same row in bf16
    # a write: rows in, codes out, codes in, values out
    return {"bytes": n * (2 * (row + plain) if kind == "write" else row + plain), "flops": 0.0}


# --------------------------------------------- the same results in 64 bits

def _code64(x, bits):
    """bf16 rows -> the values their codes stand for, by a search of the grid."""
    limit, most, low, top = CODES[bits]
    grid = torch.tensor(E2M1, dtype=F64, device=x.device) if bits == 4 else torch.arange(
        127, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).to(F64)
    x = x.to(F64).unflatten(-1, (-1, 32))
    a = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(a.clamp(min=2.0 ** -200) / limit))
    e = torch.where(a <= limit * torch.exp2(e - 1), e - 1, e)     # the logarithm's own rounding
    e = torch.where(a > limit * torch.exp2(e), e + 1, e).clamp(min=low)
    y = (x.abs() / torch.exp2(e)).clamp(max=most)
    hi = torch.searchsorted(grid, y).clamp(max=len(grid) - 1)
    lo = (hi - 1).clamp(min=0)
    up, down = grid[hi] - y, y - grid[lo]
    near = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), grid[hi], grid[lo])
    return (torch.where(x < 0, -near, near) * torch.exp2(e)).flatten(-2)


def _decode64(p, bits, layer, which, ids, h):
    """Rows [.., d] of one head of the pages ids."""
    c, s = p.codes[layer, which, ids, h], p.scales[layer, which, ids, h].to(F64)
    if bits == 8:
        x = c.view(torch.float8_e4m3fn).to(F64)
    else:
        grid = torch.tensor(E2M1, dtype=F64, device=c.device)
        x = torch.empty(*c.shape[:-1], p.d, dtype=F64, device=c.device)
        for i, nib in enumerate((c % 16, c // 16)):
            x[..., i::2] = grid[(nib % 8).long()] * (1.0 - 2.0 * (nib // 8).to(F64))
    return (x * torch.exp2(s - 127).repeat_interleave(32, -1)).reshape(-1, p.d)


def _attend64(case, seed):
    st = _prepare_attend(case, seed)
    p = st["pages"]
    hq, hkv, d = HEADS[case["heads"]]
    bits, rep = case["bits"], hq // hkv
    rows, opened, table = p.rows.tolist(), p.open.tolist(), p.table.tolist()
    o64 = torch.zeros(st["o"].shape, dtype=F64, device=DEV)
    l64 = torch.zeros(st["lse"].shape, dtype=F64, device=DEV)
    for layer in range(case["layers"]):
        for b in range(case["batch"]):
            n, m = rows[b], opened[b]
            ids = torch.tensor(table[b][:-(-n // case["page"])], device=DEV)
            for h in range(hkv):
                k, v = (_decode64(p, bits, layer, w, ids, h)[:n] for w in (0, 1))
                for j in range(h * rep, (h + 1) * rep):
                    s = st["q"][layer, b, :m, j].to(F64) @ k.t() / d ** 0.5
                    s[:, n - m:] += torch.full((m, m), -math.inf, dtype=F64, device=DEV).triu(1)
                    l64[layer, b, :m, j] = torch.logsumexp(s, 1)
                    o64[layer, b, :m, j] = torch.softmax(s, 1) @ v
    return {"o": o64, "lse": l64}


def _write64(case, seed):
    st = _prepare_rows(case, seed)
    out = {}
    for name in ("K", "V"):
        x = torch.zeros(st[name].shape, dtype=F64, device=DEV)
        for b, n in enumerate(st["n"].tolist()):
            x[b, :n] = _code64(st[name][b, :n], case["bits"])
        out[name] = x
    return out


def _read64(case, seed):
    st = _prepare_rows(case, seed)
    p, table = st["pages"], st["pages"].table.tolist()
    K, V = (torch.zeros(x.shape, dtype=F64, device=DEV) for x in st["back"])
    for b, (lo, n) in enumerate(zip(st["first"].tolist(), st["n"].tolist())):
        j = lo // p.page
        ids = torch.tensor(table[b][j:-(-(lo + n) // p.page)], device=DEV)
        for layer in range(case["layers"]):
            for h in range(p.hkv):
                for w, x in ((0, K), (1, V)):
                    rows = _decode64(p, case["bits"], layer, w, ids, h)
                    x[b, :n, layer, h] = rows[lo - j * p.page:][:n]
    return {"K": K, "V": V}


def _logprobs64(case, seed):
    st = _prepare_logprobs(case, seed)
    b, R, V = case["batch"], case["rows"], case["vocab"]
    counts = st["n"].tolist() if st["n"] is not None else [R] * b
    logp, ent = (torch.zeros(b, R, dtype=F64, device=DEV) for _ in range(2))
    top = torch.zeros(b, R, case["top"], dtype=F64, device=DEV)
    for i in range(b):
        for r in range(counts[i]):
            lp = torch.log_softmax(st["z"][i, r].to(F64) / case["temperature"], 0)
            logp[i, r] = lp[st["y"][i, r].long()]
            ent[i, r] = -(lp.exp() * lp).sum()
            top[i, r] = torch.topk(lp, case["top"])[0]
    return (logp, ent, None, None, top)


def exact(case, seed):
    """From the definitions: attention head by head, the codes of written rows by a
    search of the grid, read rows page by page, log probabilities row by row."""
    return {"attend": _attend64, "write": _write64, "read": _read64,
            "logprobs": _logprobs64}[case["kind"]](case, seed)
