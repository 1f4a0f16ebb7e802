"""The key/value cache in 8 bits and the attention that reads it: what is measured of them.

A cache holds keys and values as 8-bit codes in pages (blocks of tokens) with one scale for each page and head:

  k        [pages][heads][page][d]   int8 or float8_e4m3fn
  v        [pages][heads][d][page]   the same, dims first
  k_scale  [pages][heads]            float32, value = code * scale; v_scale likewise

Sequence b's position p lies in page table[b][p // page].  The rows of a call (new keys, rows read back, queries) are
packed over the sequences: rows starts[b] .. starts[b + 1] are its last positions, up to lens[b].

The kinds of pass:
  write   kv_write of new rows, then kv_read of every page that they touched: what the codes now stand for
  read    kv_read of the last rows of every sequence
  attend  kv_attend of queries at the last positions of every sequence, with the log-sum-exp of their scores

Where `own` is false the same is computed by elementary torch operations in 32 bits.
"""
import math
import random

import torch

own = False

DEV = "cuda"
TYPES = {"bf16": torch.bfloat16, "f16": torch.float16}
CODES = {"int8": torch.int8, "fp8": torch.float8_e4m3fn}
QMAX = {"int8": 127.0, "fp8": 448.0}
SCORES = 1 << 28  # scores held at a time by the plain form


# ---- the cases ---------------------------------------------------------------------------------------------------

def _case(name, kind, fmt, type_, page, heads, d, n, lens, rows, mix, **kw):
    c = dict(kind=kind, fmt=fmt, type=type_, page=page, heads=heads, d=d, n=n, len_lo=lens[0], len_hi=lens[1],
             row_lo=rows[0], row_hi=rows[1], mix=mix, **kw)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's next token is put into the cache: latency
        _case("append_int8_b1", "write", "int8", "bf16", 64, 8, 128, 1, (1021, 1021), (1, 1), 1),
        # a serving batch's next tokens, sequences of all ages: the open page's scale grows now and then
        _case("append_fp8_b64", "write", "fp8", "f16", 32, 8, 128, 64, (1, 8192), (1, 1), 2),
        # prompts of a batch written at once
        _case("prompt_write_int8_64k", "write", "int8", "bf16", 64, 8, 128, 8, (2000, 14000), (2000, 14000), 3),
        # a short prefix handed on in 16 bits
        _case("read_int8_b2", "read", "int8", "bf16", 64, 8, 128, 2, (300, 700), (300, 700), 4),
        # whole caches read back for another consumer (clustering of the keys, a copy to another process); odd head size
        _case("read_fp8_d96_b16", "read", "fp8", "f16", 128, 8, 96, 16, (500, 9000), (500, 9000), 5),
        # single token, short context, one sequence: latency
        _case("token_int8_b1_800", "attend", "int8", "bf16", 64, 8, 128, 1, (777, 777), (1, 1), 6, group=4),
        # single token over a long document: the whole card on one sequence
        _case("token_int8_b1_128k", "attend", "int8", "bf16", 64, 8, 128, 1, (131071, 131071), (1, 1), 7, group=4),
        # a full serving batch of ragged contexts
        _case("token_int8_b64", "attend", "int8", "bf16", 64, 8, 128, 64, (1, 16384), (1, 1), 8, group=4),
        # every query head has its own keys, small heads, small pages
        _case("token_fp8_heads16_d64_b32", "attend", "fp8", "f16", 16, 16, 64, 32, (40, 6000), (1, 1), 9, group=1),
        # a few drafted tokens checked at once, wide groups, a sliding window
        _case("check_fp8_window_b16", "attend", "fp8", "bf16", 32, 4, 128, 16, (1000, 20000), (4, 4), 10, group=8,
              window=4096),
        # the next piece of several prompts, earlier pieces in the cache; large heads
        _case("piece_int8_d256", "attend", "int8", "f16", 64, 4, 256, 4, (600, 5000), (500, 2048), 11, group=4),
        # a long prompt at once
        _case("prompt_int8_16k", "attend", "int8", "bf16", 64, 8, 128, 1, (16384, 16384), (16384, 16384), 12, group=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    what = rng.choice(["append", "prompt_write", "read", "token", "token", "token", "check", "piece", "piece"])
    fmt, type_ = rng.choice(["int8", "int8", "fp8"]), rng.choice(["bf16", "bf16", "f16"])
    page, heads = rng.choice([16, 32, 64, 64, 128]), rng.choice([1, 2, 3, 4, 8, 8, 16])
    d = rng.choice([64, 80, 96, 128, 128, 192, 256])
    mix = rng.randrange(1 << 30)
    if what in ("append", "token", "check"):
        n = _log(rng, 1, 64)
        hi = _log(rng, 16, 131072)
        rows = 1 if what != "check" else rng.randint(2, 8)
        hi = max(rows, min(hi, int(1.0e9 / (2 * n * heads * d))))
        lens = (max(rows, rng.choice([1, hi // 4, hi])), hi)
        rows = (rows, rows)
    else:
        n = rng.randint(1, 8)
        hi = max(2, min(_log(rng, 64, 12000), int(1.3e8 / (n * heads * d))))
        rows = (rng.randint(1, hi), hi)
        lens = rows if what != "piece" else (hi, hi + _log(rng, 1, 4096))
    if what in ("append", "prompt_write", "read"):
        return _case(None, "read" if what == "read" else "write", fmt, type_, page, heads, d, n, lens, rows, mix)
    group = rng.choice([1, 2, 4, 4, 5, 8, 16])
    c = _case(None, "attend", fmt, type_, page, heads, d, n, lens, rows, mix, group=group)
    if rng.random() < 0.2:
        c["window"] = _log(rng, 16, 8192)
    if what == "piece":
        if rng.random() < 0.15:
            c["causal"] = False
            c.pop("window", None)
        while c["group"] > 1 and work(c)["flops"] > 2.0e12:  # no dearer than the largest listed call
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


# ---- inputs ------------------------------------------------------------------------------------------------------

def _gen(seed, salt):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 1009 + salt)
    return g


def _codes(fmt, shape, g):
    """Codes as a full page has them: values of a normal distribution, the largest of a page near the end of the range."""
    out = torch.empty(shape, dtype=CODES[fmt], device=DEV)
    flat = out.view(-1)
    for lo in range(0, flat.numel(), 1 << 26):
        x = torch.randn(min(1 << 26, flat.numel() - lo), generator=g, device=DEV) * (QMAX[fmt] / 4)
        x = x.clamp_(-QMAX[fmt], QMAX[fmt])
        flat[lo:lo + (1 << 26)] = (x.round_() if fmt == "int8" else x).to(CODES[fmt])
    return out


def _starts(rows):
    s = [0]
    for r in rows:
        s.append(s[-1] + r)
    return s


def prepare(case, seed):
    fmt, page, heads, d, n = case["fmt"], case["page"], case["heads"], case["d"], case["n"]
    dt = TYPES[case["type"]]
    lens, rows = _sizes(case)
    g = _gen(seed, 7)
    per = [-(-l // page) for l in lens]
    wide = max(per)
    pages = sum(per) + 3  # a few that belong to nobody
    order = torch.randperm(pages, generator=g, device=DEV).tolist()
    table, at = [], 0
    for p in per:
        table.append(order[at:at + p] + [-1] * (wide - p))
        at += p
    s = dict(case, lens_host=lens, rows_host=rows, table_host=table, own=own)
    s["table"] = torch.tensor(table, dtype=torch.int32, device=DEV)
    s["lens"] = torch.tensor(lens, dtype=torch.int32, device=DEV)
    s["starts_host"] = _starts(rows)
    s["starts"] = torch.tensor(s["starts_host"], dtype=torch.int32, device=DEV)
    s["k"] = _codes(fmt, (pages, heads, page, d), g)
    s["v"] = _codes(fmt, (pages, heads, d, page), g)
    # what values of size about 1 leave: the page's largest, 3.4 to 4.6, over the largest code, 8 bits of its inverse
    for name in ("k_scale", "v_scale"):
        top = 3.4 + 1.2 * torch.rand(pages, heads, generator=g, device=DEV)
        s[name] = 1.0 / _short(QMAX[fmt] / top)
    total = s["starts_host"][-1]
    if case["kind"] == "attend":
        hq = heads * case["group"]
        s["q"] = (torch.randn(total, hq, d, generator=g, device=DEV) * 1.5).to(dt)
    elif case["kind"] == "write":
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
        import paper_2608_14648_amd as km
        s["cache"] = km.KvCache(s["k"], s["v"], s["k_scale"], s["v_scale"])
        s["seqs"] = km.KvSeqs(s["table"], s["lens"], s["starts"], rows=total, max_rows=max(rows), max_len=max(lens))
        if case["kind"] == "write":
            s["back"] = km.KvSeqs(s["table"], s["lens"], s["back_starts"], rows=sum(s["back_host"]),
                                  max_rows=max(s["back_host"]), max_len=max(lens))
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------

def _short(x):
    """x without what lies below its eight leading bits."""
    return (x.view(torch.int32) & -65536).view(torch.float32)


def _round(x, fmt):
    return x.round() if fmt == "int8" else x.to(torch.float8_e4m3fn).float()


def _plain_write(s):
    fmt, page, heads, d = s["fmt"], s["page"], s["heads"], s["d"]
    for b, (ln, r) in enumerate(zip(s["lens_host"], s["rows_host"])):
        off = (ln - r) % page
        pg = s["table"][b, (ln - r) // page:-(-ln // page)].long()
        rows = slice(s["starts_host"][b], s["starts_host"][b] + r)
        for new, codes, scale in ((s["new_k"], s["k"], s["k_scale"]), (s["new_v"], s["v"], s["v_scale"])):
            x = torch.zeros(len(pg) * page, heads, d, device=DEV)
            x[off:off + r] = new[rows].float()
            x = x.view(len(pg), page, heads, d).transpose(1, 2)  # pages, heads, page, d
            fin = torch.where(x.isfinite(), x, torch.zeros_like(x))
            top = fin.abs().amax((2, 3))
            mul = _short((QMAX[fmt] / top).clamp(max=2.0 ** 100))
            old = codes[pg].float()
            if codes is s["v"]:
                old = old.transpose(2, 3)
            if off:
                was = _short(1.0 / scale[pg[0]] * (1 + 2.0 ** -10))
                mul[0] = torch.minimum(mul[0], was)
                old[0] = _round(old[0] * mul[0, :, None, None] / was[:, None, None], fmt)
            x = torch.minimum(torch.maximum(x.nan_to_num(0.0, math.inf, -math.inf), -top[..., None, None]),
                              top[..., None, None])
            x = _round(x * mul[..., None, None], fmt)
            pos = torch.arange(len(pg) * page, device=DEV).view(len(pg), 1, page, 1)
            x = torch.where((pos >= off) & (pos < off + r), x, old).to(CODES[fmt])
            codes[pg] = x.transpose(2, 3) if codes is s["v"] else x
            scale[pg] = 1.0 / mul


def _plain_rows(s, b, n):
    """The last n rows of sequence b in 32 bits: keys and values [n][heads][d]."""
    page, ln = s["page"], s["lens_host"][b]
    first = (ln - n) // page
    pg = s["table"][b, first:-(-ln // page)].long()
    k = s["k"][pg].float() * s["k_scale"][pg][:, :, None, None]
    v = s["v"][pg].float() * s["v_scale"][pg][:, :, None, None]
    k = k.transpose(1, 2).reshape(-1, s["heads"], s["d"])
    v = v.permute(0, 3, 1, 2).reshape(-1, s["heads"], s["d"])
    lo = ln - n - first * page
    return k[lo:lo + n], v[lo:lo + n]


def _plain_read(s, rows):
    dt = TYPES[s["type"]]
    top = torch.finfo(dt).max
    got = [_plain_rows(s, b, n) for b, n in enumerate(rows)]
    return [torch.cat([x[i].clamp(-top, top) for x in got]).to(dt) for i in (0, 1)]


def _plain_attend(s):
    d, heads, group = s["d"], s["heads"], s["group"]
    causal, window = s.get("causal", True), s.get("window", 0)
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], device=DEV)
    for b, (ln, r) in enumerate(zip(s["lens_host"], s["rows_host"])):
        k, v = _plain_rows(s, b, ln)
        k, v = k.permute(1, 2, 0).contiguous(), v.transpose(0, 1).contiguous()  # heads, d, len / heads, len, d
        step = max(1, SCORES // (heads * group * ln))
        for lo in range(0, r, step):
            m = min(step, r - lo)
            at = s["starts_host"][b] + lo
            q = s["q"][at:at + m].float().view(m, heads, group, d).permute(1, 0, 2, 3).reshape(heads, m * group, d)
            p0, p1 = ln - r + lo, ln - r + lo + m  # positions of these queries
            j0 = max(0, p0 - window + 1) if window else 0
            j1 = p1 if causal else ln
            w = torch.bmm(q, k[:, :, j0:j1].contiguous()) * (1 / math.sqrt(d))
            if causal:
                pos = torch.arange(p0, p1, device=DEV).repeat_interleave(group)[:, None]
                j = torch.arange(j0, j1, device=DEV)[None]
                hide = j > pos
                if window:
                    hide |= j <= pos - window
                w.masked_fill_(hide, -math.inf)
            top = w.amax(2, keepdim=True)
            w = w.sub_(top).exp_()
            tot = w.sum(2, keepdim=True)
            o = torch.bmm(w, v[:, j0:j1].contiguous()) / tot
            out[at:at + m] = o.view(heads, m, group, d).permute(1, 0, 2, 3).reshape(m, heads * group, d).to(out.dtype)
            e = (top + tot.log()).view(heads, m, group)
            lse[at:at + m] = e.permute(1, 0, 2).reshape(m, heads * group)
    return [out, lse]


def run(s):
    kind = s["kind"]
    if s["own"]:
        import paper_2608_14648_amd as km
        if kind == "attend":
            return list(km.kv_attend(s["cache"], s["seqs"], s["q"], causal=s.get("causal", True),
                                     window=s.get("window", 0), lse=True))
        if kind == "write":
            km.kv_write(s["cache"], s["seqs"], s["new_k"], s["new_v"])
            return list(km.kv_read(s["cache"], s["back"], TYPES[s["type"]]))
        return list(km.kv_read(s["cache"], s["seqs"], TYPES[s["type"]]))
    if kind == "attend":
        return _plain_attend(s)
    if kind == "write":
        _plain_write(s)
        return _plain_read(s, s["back_host"])
    return _plain_read(s, s["rows_host"])


# ---- what a pass cannot do without -------------------------------------------------------------------------------

def work(case):
    lens, rows = _sizes(case)
    page, heads, d = case["page"], case["heads"], case["d"]
    token = 2 * heads * d  # codes of a token's key and value
    total = sum(rows)
    if case["kind"] == "attend":
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
        return {"bytes": seen * token + 8 * heads * (seen // page) + 4 * total * hq * d + 4 * total * hq,
                "flops": 4 * pairs * hq * d}
    if case["kind"] == "read":
        return {"bytes": 3 * total * token + 8 * heads * (total // page), "flops": total * token}
    back = sum(ln - (ln - r) // page * page for ln, r in zip(lens, rows))
    # new rows in, their codes out; the touched pages' earlier codes in, all of their rows out
    return {"bytes": 2 * total * token + 3 * back * token, "flops": 3 * total * token + back * token}


# ---- the same outputs in 64 bits ---------------------------------------------------------------------------------

def _exact_code(y, fmt):
    """y rounded to the nearest code, halves to the even one, in 64 bits."""
    if fmt == "int8":
        return torch.round(y)
    # e4m3: four significant bits down to 2^-6, steps of 2^-9 below
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    e = torch.where(torch.exp2(e) > y.abs().clamp(min=2.0 ** -6), e - 1, e)
    e = torch.where(torch.exp2(e + 1) <= y.abs(), e + 1, e).clamp(min=-6)
    step = torch.exp2(e - 3)
    return torch.round(y / step) * step


def _exact_seq(s, b):
    """Codes times scales of one whole sequence in 64 bits: [len][heads][d] twice."""
    page = s["page"]
    ln = s["lens_host"][b]
    pos = torch.arange(ln, device=DEV)
    pg = torch.tensor(s["table_host"][b], device=DEV)[pos // page]
    k = s["k"].view(torch.uint8)[pg, :, pos % page].view(CODES[s["fmt"]])
    v = s["v"].view(torch.uint8)[pg, :, :, pos % page].view(CODES[s["fmt"]])
    return (k.double() * s["k_scale"].double()[pg][:, :, None], v.double() * s["v_scale"].double()[pg][:, :, None])


def exact(case, seed):
    s = prepare(case, seed)
    fmt, page = case["fmt"], case["page"]
    first, second = [], []
    for b, (ln, r) in enumerate(zip(s["lens_host"], s["rows_host"])):
        if case["kind"] == "read":
            k, v = _exact_seq(s, b)
            first.append(k[ln - r:])
            second.append(v[ln - r:])
        elif case["kind"] == "write":
            k, v = _exact_seq(s, b)
            start = (ln - r) // page * page
            lo = s["starts_host"][b]
            for vals, new, scale, out in ((k, s["new_k"], s["k_scale"], first), (v, s["new_v"], s["v_scale"], second)):
                x = new[lo:lo + r].double()
                for p in range(start, ln, page):
                    i0, i1 = max(p, ln - r), min(p + page, ln)
                    part = x[i0 - (ln - r):i1 - (ln - r)]
                    top = part.abs().amax((0, 2))
                    # the multiplier has eight significant bits
                    mul = (QMAX[fmt] / top).clamp(max=2.0 ** 100)
                    e = torch.floor(torch.log2(mul)) - 7
                    mul = torch.floor(mul / torch.exp2(e)) * torch.exp2(e)
                    rows = []
                    if i0 > p:
                        sc = scale[s["table_host"][b][p // page]].double()
                        was = 1.0 / sc
                        e = torch.floor(torch.log2(was * (1 + 2.0 ** -20))) - 7
                        was = torch.round(was / torch.exp2(e)) * torch.exp2(e)
                        mul = torch.minimum(mul, was)
                        code = vals[p:i0] / sc[:, None]
                        code = code.round() if fmt == "int8" else code.float().to(CODES[fmt]).double()
                        rows.append(_exact_code(code * mul[:, None] / was[:, None], fmt))
                    rows.append(_exact_code(part * mul[:, None], fmt))
                    out.append(torch.cat(rows) / mul[:, None])
        else:
            k, v = _exact_seq(s, b)
            causal, window, heads, group = case.get("causal", True), case.get("window", 0), case["heads"], case["group"]
            lo = s["starts_host"][b]
            o = torch.empty(r, heads * group, case["d"], dtype=torch.float64, device=DEV)
            lse = torch.empty(r, heads * group, dtype=torch.float64, device=DEV)
            step = max(1, (1 << 26) // ln)
            j = torch.arange(ln, device=DEV)
            for h in range(heads * group):
                kh, vh = k[:, h // group].contiguous(), v[:, h // group].contiguous()
                for i in range(0, r, step):
                    q = s["q"][lo + i:lo + min(r, i + step), h].double()
                    z = (q @ kh.T) / math.sqrt(case["d"])
                    if causal:
                        at = (ln - r + i + torch.arange(q.shape[0], device=DEV))[:, None]
                        seen = j <= at
                        if window:
                            seen &= j > at - window
                        z = torch.where(seen, z, torch.full_like(z, -math.inf))
                    e = torch.logsumexp(z, 1)
                    lse[i:i + step, h] = e
                    o[i:i + step, h] = torch.exp(z - e[:, None]) @ vh
            first.append(o)
            second.append(lse)
    return [torch.cat(first), torch.cat(second)]
