"""What a serving program does around the key/value cache: what is measured of it.

A cache is the one of perf/operators.py, or holds 4-bit codes:

  k        [pages][heads][page][d]     int8 or float8_e4m3fn; 4 bits: uint8 [pages][heads][page][d / 2], two dims a byte
  v        [pages][heads][d][page]     the same, dims first; 4 bits: uint8 [pages][heads][d][page / 2], two tokens a byte
  k_scale  [pages][heads]              float32, value = code * scale; v_scale likewise.  4 bits: [pages][heads][page],
                                       a scale for each token and head

A 4-bit code is a whole number -7 .. 7, held as code + 8; the even dim or token is the low half of its byte.  A row of a
token and head with largest magnitude a has the multiplier 7 / a without what lies below its eight leading bits, within
[2^-30, 2^30], the code nearest to value times multiplier and the scale 1 / multiplier.

Sequence b's position p lies in page table[b][p // page].  The rows of a call are packed over the sequences: rows
starts[b] .. starts[b + 1] are its last positions, up to lens[b].

The kinds of pass:
  rotate  kv_rotate of queries and keys by their positions
  write   kv_write of new rows into a 4-bit cache, then kv_read of every page that they touched
  attend  kv_attend over a 4-bit cache, with the log-sum-exp of the scores
  weigh   kv_weigh: the attention weight that every cached token gets from the call's rows, added to what it had
  evict   kv_evict: the heaviest tokens of each sequence and head move to the front of its pages, then kv_read of them

Where `own` is false the same is computed by elementary torch operations in 32 bits (angles in 64).
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
CODES = {"int8": torch.int8, "fp8": torch.float8_e4m3fn, "int4": torch.uint8}
QMAX = {"int8": 127.0, "fp8": 448.0, "int4": 7.0}
SCORES = 1 << 28  # scores held at a time by the plain form


# ---- the cases ---------------------------------------------------------------------------------------------------

def _rotate(name, type_, layout, dims, heads, group, d, n, lens, rows, mix, **kw):
    c = dict(kind="rotate", type=type_, layout=layout, dims=dims, page=64, heads=heads, group=group, d=d, n=n,
             len_lo=lens[0], len_hi=lens[1], row_lo=rows[0], row_hi=rows[1], mix=mix, **kw)
    if name:
        c["name"] = name
    return c


def _case(name, kind, fmt, type_, page, heads, d, n, lens, rows, mix, **kw):
    c = dict(kind=kind, fmt=fmt, type=type_, page=page, heads=heads, d=d, n=n, len_lo=lens[0], len_hi=lens[1],
             row_lo=rows[0], row_hi=rows[1], mix=mix, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the next tokens of a serving batch, sequences of all ages: latency
        _rotate("rotate_tokens_b32", "bf16", "halves", 128, 8, 4, 128, 32, (1, 131072), (1, 1), 1),
        # a training batch on its way back: the gradient of four packed documents' queries and keys; half of each head turned,
        # frequencies stretched for contexts eight times as long
        _rotate("rotate_back_pairs_16k", "f16", "pairs", 64, 8, 4, 128, 4, (2500, 5500), (2500, 5500), 2, inverse=True,
                scaling="parts", factor=8.0),
        # a serving batch's next tokens are put into the cache
        _case("append_int4_b64", "write", "int4", "f16", 32, 8, 128, 64, (1, 8192), (1, 1), 3),
        # prompts of a batch written at once
        _case("prompt_write_int4_64k", "write", "int4", "bf16", 64, 8, 128, 8, (2000, 14000), (2000, 14000), 4),
        # single token, short context, one sequence: latency
        _case("token_int4_b1_900", "attend", "int4", "bf16", 64, 8, 128, 1, (901, 901), (1, 1), 5, group=4),
        # single token over a long document: the whole card on one sequence; odd head size, small pages
        _case("token_int4_d96_b1_128k", "attend", "int4", "f16", 16, 8, 96, 1, (131071, 131071), (1, 1), 6, group=6),
        # a full serving batch of ragged contexts
        _case("token_int4_b64", "attend", "int4", "bf16", 64, 8, 128, 64, (1, 16384), (1, 1), 7, group=4),
        # the next piece of several prompts, earlier pieces in the cache
        _case("piece_int4_b4", "attend", "int4", "bf16", 64, 8, 128, 4, (3000, 12000), (1000, 4096), 8, group=4),
        # a serving batch's single tokens add their weights to those of an int8 cache
        _case("weigh_tokens_int8_b16", "weigh", "int8", "bf16", 64, 8, 128, 16, (500, 8192), (1, 1), 9, group=4),
        # two prompts' weights, all of their rows
        _case("weigh_prompts_int4", "weigh", "int4", "f16", 64, 8, 128, 2, (3000, 6000), (3000, 6000), 10, group=4),
        # contexts past their budget are halved
        _case("evict_int8_b8", "evict", "int8", "bf16", 64, 8, 128, 8, (3900, 4300), (0, 0), 11, keep=2048, first=4,
              recent=64),
        # a long document cut down to what its reader looked at
        _case("evict_int4_b1_100k", "evict", "int4", "bf16", 64, 8, 128, 1, (100001, 100001), (0, 0), 12, keep=8192, first=4,
              recent=128),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["rotate", "rotate", "append", "prompt_write", "token", "token", "check", "piece", "weigh", "weigh",
                       "evict", "evict"])
    type_ = rng.choice(["bf16", "bf16", "f16"])
    page, heads = rng.choice([16, 32, 64, 64, 128]), rng.choice([1, 2, 3, 4, 8, 8, 16])
    mix = rng.randrange(1 << 30)
    if what == "rotate":
        d = rng.choice([64, 80, 96, 128, 128, 192, 256])
        group = rng.choice([1, 2, 4, 4, 5, 8])
        dims = rng.choice([d, d, d // 2, d // 4])
        n = _log(rng, 1, 64)
        one = rng.random() < 0.4
        hi = 1 if one else max(2, min(_log(rng, 2, 8192), int(8.0e7 / (n * heads * (group + 1) * d))))
        rows = (1, 1) if one else (rng.randint(1, hi), hi)
        far = _log(rng, hi, 1 << 20)
        kw = dict(inverse=True) if rng.random() < 0.4 else {}
        how = rng.choice([None, None, "linear", "base", "parts"])
        if how:
            kw.update(scaling=how, factor=rng.choice([2.0, 4.0, 8.0, 32.0]))
        return _rotate(None, rng.choice(["bf16", "f16", "f32"]), rng.choice(["halves", "pairs"]), dims, heads, group, d, n,
                       (rows[0], far), rows, mix, **kw)
    d = rng.choice([64, 96, 128, 128, 160, 192, 256])
    fmt = rng.choice(["int4", "int4", "int8", "fp8"]) if what in ("weigh", "evict") else "int4"
    if what == "append":
        n = _log(rng, 1, 64)
        hi = max(1, min(_log(rng, 16, 32768), int(1.0e9 / (2 * n * heads * d))))
        return _case(None, "write", fmt, type_, page, heads, d, n, (1, hi), (1, 1), mix)
    if what == "prompt_write":
        n = rng.randint(1, 8)
        hi = max(2, min(_log(rng, 64, 12000), int(7.5e7 / (n * heads * d))))
        rows = (rng.randint(1, hi), hi)
        return _case(None, "write", fmt, type_, page, heads, d, n, rows, rows, mix)
    if what == "evict":
        n = _log(rng, 1, 16)
        hi = max(40, min(_log(rng, 64, 100000), int(1.0e8 / (n * heads * d))))
        return _case(None, "evict", fmt, type_, page, heads, d, n, (hi // 2, hi), (0, 0), mix,
                     keep=rng.randint(16, max(16, int(hi * rng.choice([0.1, 0.3, 0.6, 1.1])))), first=rng.choice([0, 4]),
                     recent=rng.choice([0, 8]))
    group = rng.choice([1, 2, 4, 4, 5, 8, 16])
    kind = "weigh" if what == "weigh" else "attend"
    if what in ("token", "check") or (what == "weigh" and rng.random() < 0.5):
        n = _log(rng, 1, 64)
        rows = rng.randint(2, 8) if what == "check" else 1
        hi = max(rows, min(_log(rng, 16, 131072), int(1.0e9 / (2 * n * heads * d))))
        lens, rows = (max(rows, rng.choice([1, hi // 4, hi])), hi), (rows, rows)
    else:
        n = rng.randint(1, 6)
        hi = max(2, min(_log(rng, 64, 5000), int(1.0e8 / (n * heads * d))))
        rows = (rng.randint(1, hi), hi)
        lens = (hi, hi + _log(rng, 1, 4096))
    c = _case(None, kind, fmt, type_, page, heads, d, n, lens, rows, mix, group=group)
    if rng.random() < 0.2:
        c["window"] = _log(rng, 16, 8192)
    elif rng.random() < 0.15:
        c["causal"] = False
    if kind == "weigh":
        c["decay"] = rng.choice([1.0, 1.0, 0.9, 0.0])
    while c["group"] > 1 and work(c)["flops"] > 2.0e11:  # no dearer than the largest listed call
        c["group"] -= 1
    return c


def _sizes(case):
    """Lengths of the sequences and the rows of each, a fixed mix that belongs to the case."""
    rng = random.Random(case["mix"])
    rows = [rng.randint(case["row_lo"], case["row_hi"]) for _ in range(case["n"])]
    lens = [rng.randint(case["len_lo"], case["len_hi"]) for _ in range(case["n"])]
    if case["row_lo"] == case["len_lo"] and case["row_hi"] == case["len_hi"] and case["row_hi"] > 1:
        lens = rows  # whole sequences
    return lens, [min(r, l) for r, l in zip(rows, lens)]


def _kept(case):
    return [min(case["keep"], l) for l in _sizes(case)[0]]


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1009 + salt)
    return g


def _codes(fmt, shape, g):
    """Codes of values of a normal distribution, the largest of a page or row near the end of the range."""
    out = torch.empty(shape, dtype=CODES[fmt], device=DEV)
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        n = min(1 << 26, flat.numel() - lo)
        if fmt == "int4":
            x = (torch.randn(2, n, generator=g, device=DEV) * 2.6).round_().clamp_(-7, 7).add_(8).to(torch.uint8)
            flat[lo:lo + n] = x[0] | (x[1] << 4)
            continue
        x = (torch.randn(n, generator=g, device=DEV) * (QMAX[fmt] / 4)).clamp_(-QMAX[fmt], QMAX[fmt])
        flat[lo:lo + n] = (x.round_() if fmt == "int8" else x).to(CODES[fmt])
    return out


def _starts(rows):
    s = [0]
    for r in rows:
        s.append(s[-1] + r)
    return s


def _frequencies(case):
    """Radians per position of each pair, 64 bits."""
    dims, base, factor = case["dims"], 10000.0, case.get("factor", 1.0)
    how, original = case.get("scaling"), 8192
    if how == "base":
        base *= factor ** (dims / max(dims - 2, 1))
    out = []
    for i in range(dims // 2):
        f = base ** (-2.0 * i / dims)
        if how == "linear":
            f /= factor
        elif how == "parts":  # pairs that turn less than once within the original length are stretched, fast ones stay
            keep = min(max((original * f / (2 * math.pi) - 1.0) / 31.0, 0.0), 1.0)
            f = f * keep + f / factor * (1 - keep)
        out.append(f)
    return out


def _lse(s):
    """The log-sum-exp that the attention of these rows has left behind."""
    out = torch.empty(s["starts_host"][-1], s["heads"] * s["group"], device=DEV)
    for b, lo, m, at, w in _scores(s):
        e = torch.logsumexp(w, 2).view(s["heads"], m, s["group"])
        out[at:at + m] = e.permute(1, 0, 2).reshape(m, -1)
    return out


def prepare(case, seed):
    page, heads, d, n, kind = case["page"], case["heads"], case["d"], case["n"], case["kind"]
    dt = TYPES[case["type"]]
    lens, rows = _sizes(case)
    g = _gen(seed, 7)
    s = dict(case, lens_host=lens, rows_host=rows, own=own)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["starts_host"] = _starts(rows)
    s["starts"] = torch.tensor(s["starts_host"], dtype=torch.int32, device=DEV)
    total = s["starts_host"][-1]
    per = [-(-l // page) for l in lens]
    wide = max(per)
    pages = sum(per) + 3  # a few that belong to nobody
    order = torch.randperm(pages, generator=g, device=DEV).tolist()
    table, at = [], 0
    for p in per:
        table.append(order[at:at + p] + [-1] * (wide - p))
        at += p
    s["table_host"] = table
    s["table"] = torch.tensor(table, dtype=torch.int32, device=DEV)
    if own:
        import paper_2608_14648_amd as km
        s["seqs"] = km.KvSeqs(s["table"], s["lens"], s["starts"], rows=total, max_rows=max(rows), max_len=max(lens))
    if kind == "rotate":
        hq = heads * case["group"]
        s["q"] = torch.randn(total, hq, d, generator=g, device=DEV).to(dt)
        s["k"] = torch.randn(total, heads, d, generator=g, device=DEV).to(dt)
        s["freq"] = torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
        first = [l - r for l, r in zip(lens, rows)]
        s["positions"] = torch.cat([torch.arange(f, f + r, device=DEV) for f, r in zip(first, rows)])
        if own:
            s["rotary"] = km.kv_rotary(case["dims"], 10000.0, layout=case["layout"], scaling=case.get("scaling"),
                                       factor=case.get("factor", 1.0), original=8192)
        return s
    fmt = case["fmt"]
    half = 2 if fmt == "int4" else 1
    s["k"] = _codes(fmt, (pages, heads, page, d // half), g)
    s["v"] = _codes(fmt, (pages, heads, d, page // half), g)
    for name in ("k_scale", "v_scale"):
        # what values of size about 1 leave: the largest over the largest code, 8 bits of its inverse
        if fmt == "int4":
            top = 2.0 + 1.4 * torch.rand(pages, heads, page, generator=g, device=DEV)
        else:
            top = 3.4 + 1.2 * torch.rand(pages, heads, generator=g, device=DEV)
        s[name] = 1.0 / _short(QMAX[fmt] / top)
    if kind in ("attend", "weigh"):
        s["q"] = (torch.randn(total, heads * case["group"], d, generator=g, device=DEV) * 1.5).to(dt)
    if kind in ("weigh", "evict"):  # weights as many rows leave them: few tokens have most
        s["weight"] = torch.exp(2.0 * torch.randn(pages, heads, page, generator=g, device=DEV))
        # some have the same
        s["weight"] = torch.where(s["weight"] < 0.3, (s["weight"] * 32).floor() / 32, s["weight"])
    if kind == "weigh":
        s["lse"] = _lse(s)
    elif kind == "evict":
        kept = _kept(case)
        s["keep_lens"] = torch.full((n,), case["keep"], dtype=torch.int32, device=DEV)
        s["left_lens"] = torch.tensor(kept, dtype=torch.int32, device=DEV)
        s["left_starts"] = torch.tensor(_starts(kept), dtype=torch.int32, device=DEV)
        s["left_host"] = kept
    elif kind == "write":
        # keys have a few large channels, and tokens differ in size
        chan = 1 + 2 * (torch.rand(2, heads, d, generator=g, device=DEV) < 0.03).float()
        for i, name in enumerate(("new_k", "new_v")):
            x = torch.randn(total, heads, d, generator=g, device=DEV)
            x *= torch.exp(0.2 * torch.randn(total, heads, 1, generator=g, device=DEV))
            s[name] = (x * chan[i]).to(dt)
        # the touched pages, from their first token
        back = [l - (l - r) // page * page for l, r in zip(lens, rows)]
        s["back_host"] = back
        s["back_starts"] = torch.tensor(_starts(back), dtype=torch.int32, device=DEV)
    if own:
        s["cache"] = km.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        if kind == "write":
            s["back"] = km.KvSeqs(s["table"], s["lens"], s["back_starts"], rows=sum(s["back_host"]),
                                  max_rows=max(s["back_host"]), max_len=max(lens))
        elif kind == "evict":
            s["left"] = km.KvSeqs(s["table"], s["left_lens"], s["left_starts"], rows=sum(kept), max_rows=max(kept),
                                  max_len=max(kept))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def _short(x):
    """x without what lies below its eight leading bits."""
    return (x.view(torch.int32) & -65536).view(torch.float32)


def _round(x, fmt):
    return x.to(torch.float8_e4m3fn).float() if fmt == "fp8" else x.round()


def _unpack(x):
    """Code values of packed 4-bit codes, the last axis twice as long."""
    return torch.stack([x & 15, x >> 4], -1).flatten(-2).float() - 8


def _pack(x):
    x = (x + 8).to(torch.uint8)
    return x[..., 0::2] | (x[..., 1::2] << 4)


def _page_codes(s, name, pg):
    """Code values of pages pg, [page][heads][token][d], and their multiplicators for each token, [page][heads][token]."""
    x = s[name][pg]
    x = _unpack(x) if s["fmt"] == "int4" else x.float()
    scale = s[name + "_scale"][pg]
    if s["fmt"] != "int4":
        scale = scale[:, :, None].expand(-1, -1, s["page"])
    return (x.transpose(2, 3) if name == "v" else x), scale


def _put_codes(s, name, pg, x):
    """The other way round."""
    if name == "v":
        x = x.transpose(2, 3)
    s[name][pg] = _pack(x) if s["fmt"] == "int4" else x.contiguous().to(CODES[s["fmt"]])


def _plain_rotate(s):
    dims, dt = s["dims"], TYPES[s["type"]]
    angle = s["positions"].double()[:, None] * s["freq"]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    if s.get("inverse"):
        sin = -sin
    out = []
    for x in (s["q"].float(), s["k"].float()):
        if s["layout"] == "halves":
            a, b = x[..., :dims // 2], x[..., dims // 2:dims]
            y = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
        else:
            a, b = x[..., 0:dims:2], x[..., 1:dims:2]
            y = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
        out.append(torch.cat([y, x[..., dims:]], -1).to(dt))
    return out


def _plain_write(s):
    page, heads, d = s["page"], s["heads"], s["d"]
    for b, (ln, r) in enumerate(zip(s["lens_host"], s["rows_host"])):
        off = (ln - r) % page
        pg = s["table"][b, (ln - r) // page:-(-ln // page)].long()
        rows = slice(s["starts_host"][b], s["starts_host"][b] + r)
        for new, name in ((s["new_k"], "k"), (s["new_v"], "v")):
            x = new[rows].float()
            fin = torch.where(x.isfinite(), x, torch.zeros_like(x))
            top = fin.abs().amax(2, keepdim=True)
            mul = _short((QMAX["int4"] / top).clamp(2.0 ** -30, 2.0 ** 30))
            x = torch.minimum(torch.maximum(x.nan_to_num(0.0, math.inf, -math.inf), -top), top)
            x = (x * mul).round().clamp(-7, 7)
            old, scale = _page_codes(s, name, pg)  # pages, heads, page, d
            old = old.transpose(1, 2).reshape(len(pg) * page, heads, d)
            scale = scale.transpose(1, 2).reshape(len(pg) * page, heads)
            old[off:off + r] = x
            scale[off:off + r] = 1.0 / mul[..., 0]
            _put_codes(s, name, pg, old.view(len(pg), page, heads, d).transpose(1, 2))
            s[name + "_scale"][pg] = scale.view(len(pg), page, heads).transpose(1, 2)


def _plain_rows(s, b, ln, n):
    """The n rows before position ln of sequence b in 32 bits: keys and values [n][heads][d]."""
    page = s["page"]
    first = (ln - n) // page
    pg = s["table"][b, first:-(-ln // page)].long()
    out = []
    for name in ("k", "v"):
        x, scale = _page_codes(s, name, pg)
        x = (x * scale[..., None]).transpose(1, 2).reshape(-1, s["heads"], s["d"])
        out.append(x[ln - n - first * page:ln - first * page])
    return out


def _plain_read(s, lens, rows):
    dt = TYPES[s["type"]]
    top = torch.finfo(dt).max
    got = [_plain_rows(s, b, ln, n) for b, (ln, n) in enumerate(zip(lens, rows))]
    return [torch.cat([x[i].clamp(-top, top) for x in got]).to(dt) for i in (0, 1)]


def _scores(s, after=None):
    """Scores of a piece of a sequence's rows at a time, [heads][rows * group][positions]: sequence, first row of it, rows,
    first row of the call, scores.  after: what is left of a sequence's values is put there."""
    d, heads, group = s["d"], s["heads"], s["group"]
    causal, window = s.get("causal", True), s.get("window", 0)
    for b, (ln, r) in enumerate(zip(s["lens_host"], s["rows_host"])):
        k, v = _plain_rows(s, b, ln, ln)
        k = k.permute(1, 2, 0).contiguous()  # heads, d, len
        if after is not None:
            after["v"] = v.transpose(0, 1).contiguous()  # heads, len, d
        del v
        step = max(1, SCORES // (heads * group * ln))
        for lo in range(0, r, step):
            m = min(step, r - lo)
            at = s["starts_host"][b] + lo
            q = s["q"][at:at + m].float().view(m, heads, group, d).permute(1, 0, 2, 3).reshape(heads, m * group, d)
            w = torch.bmm(q, k) * (1 / math.sqrt(d))
            if causal:
                pos = torch.arange(ln - r + lo, ln - r + lo + m, device=DEV).repeat_interleave(group)[:, None]
                j = torch.arange(ln, device=DEV)[None]
                hide = j > pos
                if window:
                    hide |= j <= pos - window
                w.masked_fill_(hide, -math.inf)
            yield b, lo, m, at, w


def _plain_attend(s):
    heads, group, d = s["heads"], s["group"], s["d"]
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], device=DEV)
    after = {}
    for b, lo, m, at, w in _scores(s, after):
        top = w.amax(2, keepdim=True)
        w = w.sub_(top).exp_()
        tot = w.sum(2, keepdim=True)
        o = torch.bmm(w, after["v"]) / tot
        out[at:at + m] = o.view(heads, m, group, d).permute(1, 0, 2, 3).reshape(m, heads * group, d).to(out.dtype)
        e = (top + tot.log()).view(heads, m, group)
        lse[at:at + m] = e.permute(1, 0, 2).reshape(m, heads * group)
    return [out, lse]


def _plain_weigh(s):
    page, heads, group, decay = s["page"], s["heads"], s["group"], s.get("decay", 1.0)
    for b, lo, m, at, w in _scores(s):
        ln, r = s["lens_host"][b], s["rows_host"][b]
        if lo == 0:
            total = torch.zeros(heads, ln, device=DEV)
        e = s["lse"][at:at + m].view(m, heads, group).permute(1, 0, 2).reshape(heads, m * group, 1)
        total += w.sub_(e).exp_().sum(1)
        if lo + m == r:
            pg = s["table"][b, :-(-ln // page)].long()
            old = s["weight"][pg].transpose(0, 1).reshape(heads, -1)
            new = old[:, :ln] * decay if decay else torch.zeros_like(total)
            new[:, ln - r:] = 0  # the call's own tokens begin with it
            old[:, :ln] = new + total
            s["weight"][pg] = old.view(heads, len(pg), page).transpose(0, 1)
    return [s["weight"]]


def _plain_evict(s):
    fmt, page, heads, keep, first, recent = s["fmt"], s["page"], s["heads"], s["keep"], s["first"], s["recent"]
    kept = torch.full((s["n"], heads, keep), -1, dtype=torch.int32, device=DEV)
    for b, ln in enumerate(s["lens_host"]):
        pg = s["table"][b, :-(-ln // page)].long()
        weight = s["weight"][pg].transpose(0, 1).reshape(heads, -1)
        key = weight[:, :ln].clone()
        key[:, :first] = math.inf
        if recent:
            key[:, max(ln - recent, 0):] = math.inf
        n = min(keep, ln)
        idx = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :n].sort(1).values
        kept[b, :, :n] = idx.int()
        to = pg[:-(-n // page)]
        room = len(to) * page
        for name in ("k", "v"):
            x, scale = _page_codes(s, name, pg)
            x = x.transpose(0, 1).reshape(heads, -1, s["d"])
            scale = scale.transpose(0, 1).reshape(heads, -1)
            got = x.gather(1, idx[:, :, None].expand(-1, -1, s["d"]))
            had = scale.gather(1, idx)
            if fmt == "int4":
                s[name + "_scale"][to] = torch.cat([had, scale[:, n:room]], 1).view(heads, -1, page).transpose(0, 1)
            else:  # one scale per page: the largest of its tokens'; the others' codes are coded again
                mul = _short(1.0 / had * (1 + 2.0 ** -10))
                pad = torch.full((heads, room - n), math.inf, device=DEV)
                least = torch.cat([mul, pad], 1).view(heads, -1, page).amin(2)
                to_mul = least.repeat_interleave(page, 1)[:, :n, None]
                got = torch.where(mul[..., None] == to_mul, got, _round(got * to_mul / mul[..., None], fmt))
                s[name + "_scale"][to] = (1.0 / least).transpose(0, 1)
            x[:, :n] = got
            _put_codes(s, name, to, x[:, :room].view(heads, -1, page, s["d"]).transpose(0, 1))
        weight[:, :n] = weight.gather(1, idx)
        s["weight"][pg] = weight.view(heads, -1, page).transpose(0, 1)
    lens = torch.tensor(s["left_host"], dtype=torch.int32, device=DEV)
    return [kept, lens, s["weight"]]


def run(s):
    kind = s["kind"]
    if s["own"]:
        import paper_2608_14648_amd as km
        if kind == "rotate":
            return list(km.kv_rotate(s["rotary"], s["seqs"], s["q"], s["k"], inverse=s.get("inverse", False)))
        if kind == "attend":
            return list(km.kv_attend(s["cache"], s["seqs"], s["q"], causal=s.get("causal", True),
                                     window=s.get("window", 0), lse=True))
        if kind == "write":
            km.kv_write(s["cache"], s["seqs"], s["new_k"], s["new_v"])
            return list(km.kv_read(s["cache"], s["back"], TYPES[s["type"]]))
        if kind == "weigh":
            km.kv_weigh(s["cache"], s["seqs"], s["q"], s["lse"], s["weight"], causal=s.get("causal", True),
                        window=s.get("window", 0), decay=s.get("decay", 1.0))
            return [s["weight"]]
        kept, lens = km.kv_evict(s["cache"], s["seqs"], s["weight"], s["keep_lens"], s["keep"], first=s["first"],
                                 recent=s["recent"])
        return [kept, lens, s["weight"]] + list(km.kv_read(s["cache"], s["left"], TYPES[s["type"]]))
    if kind == "rotate":
        return _plain_rotate(s)
    if kind == "attend":
        return _plain_attend(s)
    if kind == "write":
        _plain_write(s)
        return _plain_read(s, s["lens_host"], s["back_host"])
    if kind == "weigh":
        return _plain_weigh(s)
    return _plain_evict(s) + _plain_read(s, s["left_host"], s["left_host"])


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    lens, rows = _sizes(case)
    kind, page, heads, d = case["kind"], case["page"], case["heads"], case["d"]
    total = sum(rows)
    elem = 4 if case["type"] == "f32" else 2
    if kind == "rotate":
        n = total * heads * (case["group"] + 1)
        return {"bytes": 2 * n * d * elem, "flops": 3 * n * case["dims"]}
    # bytes of a token's key or value and its scale, in all heads
    token = heads * (d // 2 + 4) if case["fmt"] == "int4" else heads * d
    if kind in ("attend", "weigh"):
        window = case.get("window", 0)
        pairs = seen = 0
        for ln, r in zip(lens, rows):
            lo = max(0, ln - r + 1 - window) if window else 0
            seen += ln - lo
            if not case.get("causal", True):
                pairs += r * ln
            elif window:
                pairs += sum(min(window, p + 1) for p in range(ln - r, ln))
            else:
                pairs += (ln - r + 1 + ln) * r // 2
        hq = heads * case["group"]
        if kind == "weigh":
            return {"bytes": seen * (token + 8 * heads) + total * hq * (elem * d + 4), "flops": 2 * pairs * hq * d}
        return {"bytes": 2 * seen * token + 2 * elem * total * hq * d + 4 * total * hq, "flops": 4 * pairs * hq * d}
    if kind == "write":
        back = sum(ln - (ln - r) // page * page for ln, r in zip(lens, rows))
        # new rows in, their codes out; the touched pages' earlier codes in, all of their rows out
        return {"bytes": 2 * total * (elem * heads * d + token) + 2 * (back - total) * token + 2 * back * elem * heads * d,
                "flops": 4 * total * heads * d + 2 * back * heads * d}
    kept = sum(_kept(case))
    # all weights in; the kept tokens' codes in and out, their weights, positions and rows out
    return {"bytes": 4 * sum(lens) * heads + 4 * kept * token + 8 * kept * heads + 2 * kept * elem * heads * d,
            "flops": sum(lens) * heads + 2 * kept * heads * d}


# ---- the same outputs in 64 bits ---------------------------------------------------------------------------------

def _exact_code(y, fmt):
    """y rounded to the nearest code, halves to the even one, in 64 bits."""
    if fmt != "fp8":
        return torch.round(y)
    # e4m3: four significant bits down to 2^-6, steps of 2^-9 below
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    e = torch.where(torch.exp2(e) > y.abs().clamp(min=2.0 ** -6), e - 1, e)
    e = torch.where(torch.exp2(e + 1) <= y.abs(), e + 1, e).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(y / step) * step


def _exact_token(s, b, which):
    """Codes of a whole sequence's keys or values, [len][heads][d], and their scales, [len][heads], in 64 bits."""
    page, ln, fmt = s["page"], s["lens_host"][b], s["fmt"]
    pos = torch.arange(ln, device=DEV)
    pg = torch.tensor(s["table_host"][b], device=DEV)[pos // page]
    at = pos % page
    raw = s[which].view(torch.uint8)
    if fmt == "int4":
        if which == "k":
            x = raw[pg, :, at]
            x = torch.stack([x % 16, x // 16], 3).reshape(ln, s["heads"], s["d"])
        else:
            x = raw[pg, :, :, at // 2]
            x = torch.where((at % 2 == 1)[:, None, None], x // 16, x % 16)
        return x.double() - 8, s[which + "_scale"].double()[pg, :, at]
    x = raw[pg, :, at] if which == "k" else raw[pg, :, :, at]
    return x.view(CODES[fmt]).double(), s[which + "_scale"].double()[pg]


def _eight_bits(x):
    e = torch.floor(torch.log2(x)) - 7
    return torch.floor(x / torch.exp2(e)) * torch.exp2(e)


def _exact_rotate(case, s):
    dims, out = case["dims"], []
    freq = torch.tensor(_frequencies(case), dtype=torch.float64, device=DEV)
    sign = -1.0 if case.get("inverse") else 1.0
    for name in ("q", "k"):
        x = s[name].double()
        y = x.clone()
        for b, (ln, r) in enumerate(zip(s["lens_host"], s["rows_host"])):
            rows = slice(s["starts_host"][b], s["starts_host"][b] + r)
            turn = torch.polar(torch.ones(1, dtype=torch.float64, device=DEV),
                               sign * torch.arange(ln - r, ln, device=DEV, dtype=torch.float64)[:, None] * freq)[:, None]
            if case["layout"] == "halves":
                i, j = torch.arange(dims // 2, device=DEV), torch.arange(dims // 2, dims, device=DEV)
            else:
                i, j = torch.arange(0, dims, 2, device=DEV), torch.arange(1, dims, 2, device=DEV)
            z = torch.complex(x[rows][..., i], x[rows][..., j]) * turn
            part = y[rows]
            part[..., i], part[..., j] = z.real, z.imag
        out.append(y)
    return out


def _exact_write(s, page):
    first, second = [], []
    for b, (ln, r) in enumerate(zip(s["lens_host"], s["rows_host"])):
        start = (ln - r) // page * page
        lo = s["starts_host"][b]
        for which, new, out in (("k", s["new_k"], first), ("v", s["new_v"], second)):
            codes, scale = _exact_token(s, b, which)
            out.append((codes * scale[:, :, None])[start:ln - r])
            x = new[lo:lo + r].double()
            mul = _eight_bits((7.0 / x.abs().amax(2)).clamp(2.0 ** -30, 2.0 ** 30))[:, :, None]
            out.append(_exact_code(x * mul, "int4").clamp(-7, 7) / mul)
    return [torch.cat(first), torch.cat(second)]


def _exact_evict(case, s):
    fmt, page, heads = case["fmt"], case["page"], case["heads"]
    kept = torch.full((case["n"], heads, case["keep"]), -1, dtype=torch.int32)
    weight = s["weight"].double()
    new_weight = weight.clone()
    rows = {"k": [], "v": []}
    for b, ln in enumerate(s["lens_host"]):
        n = min(case["keep"], ln)
        pos = torch.arange(ln, device=DEV)
        pg = torch.tensor(s["table_host"][b], device=DEV)[pos // page]
        tokens = {w: _exact_token(s, b, w) for w in ("k", "v")}
        got = {w: torch.empty(n, heads, case["d"], dtype=torch.float64, device=DEV) for w in ("k", "v")}
        for h in range(heads):
            w = weight[pg, h, pos % page].cpu().tolist()
            last = ln - case["recent"] if case["recent"] else ln
            order = sorted(range(ln), key=lambda j: (0, 0.0, j) if j < case["first"] or j >= last else (1, -w[j], j))
            idx = torch.tensor(sorted(order[:n]), device=DEV)
            kept[b, h, :n] = idx.int().cpu()
            slot = torch.arange(n, device=DEV)
            new_weight[pg[slot], h, slot % page] = weight[pg[idx], h, idx % page]
            for which in ("k", "v"):
                codes, scale = tokens[which]
                c, sc = codes[idx, h], scale[idx, h]
                if fmt != "int4":
                    mul = 1.0 / sc
                    e = torch.floor(torch.log2(mul * (1 + 2.0 ** -20))) - 7
                    mul = torch.round(mul / torch.exp2(e)) * torch.exp2(e)
                    least = torch.full((-(-n // page),), math.inf, dtype=torch.float64, device=DEV)
                    least = least.scatter_reduce(0, slot // page, mul, "amin")[slot // page]
                    c = torch.where((mul == least)[:, None], c, _exact_code(c * least[:, None] / mul[:, None], fmt))
                    sc = 1.0 / least
                got[which][:, h] = c * sc[:, None]
        for which in ("k", "v"):
            rows[which].append(got[which])
    lens = torch.tensor([min(case["keep"], l) for l in s["lens_host"]], dtype=torch.int32)
    return [kept.to(DEV), lens.to(DEV), new_weight, torch.cat(rows["k"]), torch.cat(rows["v"])]


def exact(case, seed):
    s = prepare(case, seed)
    kind, page = case["kind"], case["page"]
    if kind == "rotate":
        return _exact_rotate(case, s)
    if kind == "write":
        return _exact_write(s, page)
    if kind == "evict":
        return _exact_evict(case, s)
    causal, window, heads, group = case.get("causal", True), case.get("window", 0), case["heads"], case["group"]
    outs, sums = [], []
    if kind == "weigh":
        weight = s["weight"].double()
    for b, (ln, r) in enumerate(zip(s["lens_host"], s["rows_host"])):
        kc, ks = _exact_token(s, b, "k")
        vc, vs = _exact_token(s, b, "v") if kind == "attend" else (None, None)
        lo = s["starts_host"][b]
        o = torch.empty(r, heads * group, case["d"] if kind == "attend" else 0, dtype=torch.float64, device=DEV)
        lse = torch.empty(r, heads * group, dtype=torch.float64, device=DEV)
        got = torch.zeros(ln, heads, dtype=torch.float64, device=DEV)
        step = max(1, (1 << 26) // ln)
        j = torch.arange(ln, device=DEV)
        for h in range(heads * group):
            kh = kc[:, h // group] * ks[:, h // group, None]
            vh = vc[:, h // group] * vs[:, h // group, None] if kind == "attend" else None
            for i in range(0, r, step):
                q = s["q"][lo + i:lo + min(r, i + step), h].double()
                z = (q @ kh.T) / math.sqrt(case["d"])
                if causal:
                    at = (ln - r + i + torch.arange(q.shape[0], device=DEV))[:, None]
                    seen = j <= at
                    if window:
                        seen &= j > at - window
                    z = torch.where(seen, z, torch.full_like(z, -math.inf))
                if kind == "weigh":
                    got[:, h // group] += torch.exp(z - s["lse"][lo + i:lo + i + q.shape[0], h, None].double()).sum(0)
                    continue
                e = torch.logsumexp(z, 1)
                lse[i:i + step, h] = e
                o[i:i + step, h] = torch.exp(z - e[:, None]) @ vh
        if kind == "weigh":
            pg = torch.tensor(s["table_host"][b], device=DEV)[j // page]
            old = weight[pg, :, j % page]
            old = torch.where((j < ln - r)[:, None], old * case.get("decay", 1.0), torch.zeros_like(old))
            weight[pg, :, j % page] = old + got
        outs.append(o)
        sums.append(lse)
    return [weight] if kind == "weigh" else [torch.cat(outs), torch.cat(sums)]
