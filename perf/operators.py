"""Performance cases of the paged cache: sequences whose tokens are kept, in 8 bits, beside the compressed cache of the low-rank policy.

Five kinds of pass, each what a serving program does in one go:

* ``store``: the new keys and values of every slot go into the cache, and the tokens come back as the values it holds (what
  hands a sequence over to ``lessdec_prefill``).
* ``attend``: attention of every slot's newest tokens over its cached ones: single tokens, chunks of prompts, both mixed; with
  a window and a few first tokens that stay visible, or over everything.
* ``fork``: the slots become copies of other slots (samples of one prompt, beams), each makes room for its next tokens, and the
  pages that are written next but still shared are copied.
* ``compact``: the pages in use move to the front of the pool, after sequences in between have gone.

A page holds ``page`` tokens of all key/value heads. A block is 16 tokens of a head: codes in e4m3 and one power of two for the
keys, one for the values, the least that keeps the block's largest magnitude within 448 (at least 2^-40, at most 2^40).
Head shapes are those of Llama 2 7B / 13B (32 / 40 heads of 128), the Falcon shape (71 query heads of 64 on one key/value head) and
grouped heads as ``bench.py --q-per-kv`` makes them; queries and keys N(0, sigma^2) with sigma ~ U[0.5, 2] per head, values N(0, 1).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 16


def _case(kind, slots, heads, dim, page, length, new=1, group=1, dtype="f16", sinks=0, window=0, ragged=False, mixed=False,
          layers=1, name=None):
    c = {} if name is None else {"name": name}
    c.update(kind=kind, slots=slots, heads=heads, dim=dim, page=page, length=length, new=new, group=group, dtype=dtype,
             sinks=sinks, window=window, ragged=ragged, mixed=mixed, layers=layers)
    return c


def listed():
    return [
        # a decode step of a small batch: one token a slot, written into blocks that are partly full
        _case("store", 4, 8, 128, 16, 777, name="store-decode-b4", ragged=True),
        # the prompts of a batch, of uneven lengths, none a multiple of a block
        _case("store", 16, 32, 128, 64, 2049, new=2049, dtype="bf16", ragged=True, name="store-prompts-b16"),
        # one interactive sequence on the 7B model: latency
        _case("attend", 1, 32, 128, 16, 1025, name="decode-7b-b1"),
        # a full batch with grouped query heads, uneven lengths up to 8192
        _case("attend", 64, 8, 128, 16, 8192, group=4, dtype="bf16", ragged=True, name="decode-gqa4-b64"),
        # one very long sequence: the work of a row spread over the chip
        _case("attend", 1, 8, 128, 64, 131072, group=5, dtype="f16", name="decode-long-b1"),
        # Falcon's 71 query heads on one key/value head, first tokens and a window of a long sequence
        _case("attend", 64, 1, 64, 32, 8192, group=71, sinks=4, window=2044, name="decode-mqa71-window"),
        # one prompt of the 7B model, causal
        _case("attend", 1, 32, 128, 64, 8192, new=8192, dtype="f16", name="prompt-7b-8k"),
        # chunked prompts in one call with slots that decode
        _case("attend", 32, 8, 128, 16, 4096, new=512, group=4, dtype="bf16", ragged=True, mixed=True, name="mixed-gqa4-b32"),
        # prompts of the 13B model under Lambda-masking: 4 first tokens and a window
        _case("attend", 4, 40, 128, 64, 4096, new=4096, dtype="bf16", sinks=4, window=820, name="prompt-13b-lambda"),
        # 64 beams of uneven parents, a token each
        _case("fork", 64, 8, 128, 16, 2050, layers=4, name="fork-beams-64"),
        # four samples of each prompt go on with a chunk of tokens
        _case("fork", 16, 32, 128, 64, 1000, new=100, layers=2, ragged=True, name="fork-samples-16"),
        # every other sequence has ended
        _case("compact", 64, 8, 128, 16, 2048, layers=4, ragged=True, name="compact-b64"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["store", "attend", "attend", "attend", "attend", "fork", "compact"])
    dim = rng.choice([128, 128, 64])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8, 16, 71 if dim == 64 else 12])
    heads = 1 if group == 71 else max(1, rng.choice([32, 40, 12, 8]) // group)
    page = rng.choice([16, 16, 32, 64, 128])
    dtype = rng.choice(["f16", "bf16"])
    ragged = rng.random() < 0.6
    sinks, window = rng.choice([(0, 0), (0, 0), (4, _log(rng, 16, 4096)), (0, _log(rng, 16, 4096)), (rng.randint(1, 70), _log(rng, 1, 700))])
    room = 64 * 8 * 128 * 4096 // (heads * dim)               # tokens in all slots: the cache of the largest listed decode step
    if kind == "store":
        slots = _log(rng, 1, 64)
        new = rng.choice([1, 1, _log(rng, 2, max(3, min(4096, room // (16 * slots))))])
        length = new + rng.choice([0, rng.randint(1, 600)])
        return _case(kind, slots, heads, dim, page, length, new, 1, dtype, ragged=ragged)
    if kind == "fork":
        slots = _log(rng, 2, 96)
        return _case(kind, slots, heads, dim, page, _log(rng, 20, max(21, min(4000, room // (16 * slots)))), rng.choice([1, 1, rng.randint(2, 200)]),
                     1, dtype, ragged=ragged, layers=rng.choice([1, 2, 4]))
    if kind == "compact":
        slots = _log(rng, 2, 64)
        return _case(kind, slots, heads, dim, page, _log(rng, 64, max(65, min(4096, room // (16 * slots)))), 1, 1, dtype, ragged=ragged,
                     layers=rng.choice([1, 2, 4]))
    if rng.random() < 0.6:                                    # a token or a few a slot
        new = rng.choice([1, 1, 1, 1, rng.randint(2, 6)])
        slots = _log(rng, 1, 128)
        length = _log(rng, 16, min(131072, room // slots))
        return _case(kind, slots, heads, dim, page, length + new, new, group, dtype, sinks, window, ragged)
    new = _log(rng, 7, 4096)
    slots = _log(rng, 1, 32)
    length = new + rng.choice([0, 0, _log(rng, 1, 8192)])
    pairs = 32 * 4096 * 4096 // (heads * group)               # query-key pairs of a head in all slots
    slots = max(1, min(slots, pairs // (new * length)))
    if new * length > pairs:
        new = max(7, pairs // length)
    return _case(kind, slots, heads, dim, page, length, new, group, dtype, sinks, window, ragged, rng.random() < 0.3)


# ---- sizes of a case, the same for every seed --------------------------------------------------------------------------

def _share(i, n):
    """Spread evenly over (0.1, 1], the last one 1."""
    return 1.0 if i == n - 1 else 0.1 + 0.9 * ((i + 1) * 0.6180339887 % 1.0)


def _rows(c):
    """(new tokens, tokens in all) of every slot; some have none."""
    n, got = c["slots"], []
    for i in range(n):
        new = c["new"]
        if c["mixed"] and i % 2:
            new = 1
        elif c["ragged"] and new > 1:
            new = 0 if i % 7 == 3 else max(1, round(new * _share(i, n)))
        length = max(new, round(c["length"] * _share(i + 5 if i < n - 1 else i, n))) if c["ragged"] else c["length"]
        got.append((new, length))
    return got


def _gone(c, new, length):
    """Pages [a, b) of a slot that no later row sees: between the first tokens and the window."""
    if not c["window"]:
        return 0, 0
    a, b = -(-c["sinks"] // c["page"]), (length - new - c["window"] + 1) // c["page"]
    return (a, b) if a < b else (0, 0)


def _pairs(c, new, length):
    """(query-key pairs, cached tokens that any row sees) of a slot and head."""
    first = length - new
    if not c["window"]:
        return new * first + new * (new + 1) // 2, length if new else 0
    w, s = c["window"], c["sinks"]
    pairs = 0
    for p in range(first, length):
        lo = max(0, p + 1 - w)
        pairs += p + 1 - lo + min(s, lo)
    lo = max(0, first + 1 - w)
    return pairs, (length - lo + min(s, lo)) if new else 0


def _parents(c):
    """What each slot becomes a copy of: beams with uneven parents, one in nine freed; or samples, four of each prompt."""
    n = c["slots"]
    if n >= 64:
        return [-1 if i % 9 == 8 else (i * i * 7 + i // 3) % n for i in range(n)]
    return [i // 4 * 4 for i in range(n)]


def work(c):
    elem, tok = 2, c["heads"] * c["dim"]
    rows = _rows(c)
    if c["kind"] == "store":
        fresh = sum(r for r, _ in rows)
        held = c["slots"] * c["new"]
        # rows read, codes written; codes read back, values written
        return {"bytes": 2 * fresh * tok * (elem + 1) + 2 * held * tok * (1 + elem), "flops": 0}
    if c["kind"] == "attend":
        got = [_pairs(c, *r) for r in rows]
        scales = c["heads"] * 2 / BLOCK
        return {"bytes": sum(t for _, t in got) * (2 * tok + scales) + 2 * elem * sum(r for r, _ in rows) * tok * c["group"],
                "flops": 4 * tok * c["group"] * sum(p for p, _ in got)}
    table = c["slots"] * 8 * (-(-(c["length"] + c["new"]) // c["page"]))
    one = c["layers"] * c["page"] * (2 * tok + c["heads"] * 2 / BLOCK)
    if c["kind"] == "fork":
        used = [f for f in _parents(c) if f >= 0]
        shared = sum(rows[f][1] % c["page"] > 0 for f in used) - len({f for f in used if rows[f][1] % c["page"]})
        return {"bytes": table + 2 * one * shared, "flops": 0}
    return {"bytes": table + 2 * one * _moved(c), "flops": 0}


def _counts(c):
    return [-(-length // c["page"]) for _, length in _rows(c)]


def _moved(c):
    """Pages that compacting moves: slots lie one behind the other and every second one is free."""
    used, at, in_use = [], 0, 0
    for i, n in enumerate(_counts(c)):
        if i % 2:
            used.append((at, at + n))
            in_use += n
        at += n
    return sum(max(0, b - max(a, in_use)) for a, b in used)


# ---- the cache's form ---------------------------------------------------------------------------------------------------

def _k_rows(codes, c):
    """[..., blocks, dim/64, 4, 16, 16] -> [..., tokens, dim]: key (token i, channel 64 h + 16 g + l) lies at [h, g, i, l]."""
    x = codes.movedim(-2, -4)
    return x.reshape(*x.shape[:-5], -1, c["dim"])


def _v_rows(codes, c):
    """[..., blocks, dim/64, 4, 16, 4, 4] -> [..., tokens, dim]: value (token 4 g + i, channel 64 h + 16 t + l) lies at [h, g, l, t, i]."""
    n = codes.dim()
    x = codes.permute(*range(n - 5), n - 4, n - 1, n - 5, n - 2, n - 3)
    return x.reshape(*x.shape[:-6], -1, c["dim"])


def _k_lay(rows, c):
    """[..., tokens, dim] -> [..., blocks, dim/64, 4, 16, 16]."""
    return rows.reshape(*rows.shape[:-2], -1, BLOCK, c["dim"] // 64, 4, 16).movedim(-4, -2)


def _v_lay(rows, c):
    x = rows.reshape(*rows.shape[:-2], -1, 4, 4, c["dim"] // 64, 4, 16)          # blocks, g, i, h, t, l
    n = x.dim()
    return x.permute(*range(n - 5), n - 3, n - 5, n - 1, n - 2, n - 4)


def _floats(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _exponent(x):
    """Of blocks [..., 16, dim]: the least e with every finite magnitude within 448 * 2^e, -40 <= e <= 40."""
    m, e = torch.frexp(torch.where(torch.isfinite(x), x.abs(), 0.0).amax((-1, -2)))
    return torch.where(m > 0, e - 9 + (m > 0.875), -40).clamp(-40, 40)


def _codes(x, e):
    """Nearest code of x / 2^e, ties to even; NaN where x is not finite."""
    y = torch.ldexp(x, -e[..., None, None]).clamp(-448, 448)
    return torch.where(torch.isfinite(x), y, math.nan).to(torch.float8_e4m3fn).view(torch.uint8)


def _shapes(c, pages):
    one = (c["layers"], pages, c["heads"], c["page"] // BLOCK, c["dim"] // 64)
    return one + (4, 16, 16), one + (4, 16, 4, 4)


def _pool(c, pages, g):
    """A pool of pages full of tokens: codes of keys and values, and their exponents [layer, page, head, block, 2]."""
    sigma = 0.5 + 1.5 * torch.rand(c["heads"], generator=g, device=DEV)
    k_shape, v_shape = _shapes(c, pages)
    k = torch.empty(k_shape, dtype=torch.uint8, device=DEV)
    v = torch.empty(v_shape, dtype=torch.uint8, device=DEV)
    e = torch.empty(*k_shape[:4], 2, dtype=torch.int8, device=DEV)
    for layer in range(c["layers"]):
        for which, to, lay in ((0, k, _k_lay), (1, v, _v_lay)):
            x = torch.randn(pages, c["heads"], c["page"] // BLOCK, BLOCK, c["dim"], generator=g, device=DEV)
            if which == 0:
                x *= sigma[:, None, None, None]
            ex = _exponent(x)
            e[layer, ..., which] = ex
            to[layer] = lay(_codes(x, ex).reshape(pages, c["heads"], c["page"], c["dim"]), c)
    return k, v, e


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 29)
    rows, page, n = _rows(c), c["page"], c["slots"]
    last = max(length for _, length in rows) + (c["new"] if c["kind"] == "fork" else 0)
    width = -(-last // page)
    table = torch.full((n, width), -1, dtype=torch.int32)
    where, count = [], 0
    for i, (new, length) in enumerate(rows):
        a, b = _gone(c, new, length) if c["kind"] == "attend" else (0, 0)
        for j in range(-(-length // page)):
            if not a <= j < b:
                where.append((i, j))
                count += 1
    spare = count // 16 + 2
    if c["kind"] == "fork":
        spare += sum(-(-(rows[f][1] + c["new"]) // page) for f in _parents(c) if f >= 0)
    pages = count + spare
    if c["kind"] == "compact":
        to = torch.arange(count)
    else:
        to = torch.randperm(pages, generator=g, device=DEV)[:count].cpu()
    if count:
        at = torch.tensor(where)
        table[at[:, 0], at[:, 1]] = to.int()
    s = {"case": c, "table": table.to(DEV), "len": _ints([length for _, length in rows])}
    refs = torch.zeros(pages, dtype=torch.int32)
    refs[to] = 1
    if c["kind"] == "compact":
        for i in range(0, n, 2):                              # the sequences that have ended
            refs[table[i][table[i] >= 0].long()] = 0
            table[i] = -1
            s["len"][i] = 0
        s["table"] = table.to(DEV)
    s["refs"] = refs.to(DEV)
    s["k"], s["v"], s["exps"] = _pool(c, pages, g)
    t = TYPES[c["dtype"]]
    behind = 3                                                # rows that belong to no slot
    starts = [0]
    for new, _ in rows:
        starts.append(starts[-1] + new)
    s["start"] = _ints(starts)
    total = starts[-1] + behind
    if c["kind"] == "store":
        for name in ("new_k", "new_v"):
            s[name] = torch.randn(total, c["heads"], c["dim"], generator=g, device=DEV).to(t)
        s["slots"] = _ints(list(range(n)))
        s["out_k"], s["out_v"] = (torch.zeros(n, c["heads"], c["new"], c["dim"], dtype=t, device=DEV) for _ in range(2))
    elif c["kind"] == "attend":
        sigma = 0.5 + 1.5 * torch.rand(c["heads"] * c["group"], 1, generator=g, device=DEV)
        s["q"] = (torch.randn(total, c["heads"] * c["group"], c["dim"], generator=g, device=DEV) * sigma).to(t)
        s["out"] = torch.zeros_like(s["q"])
    elif c["kind"] == "fork":
        s["from"] = _ints(_parents(c))
        s["wanted"] = _ints([c["new"] if f >= 0 else 0 for f in _parents(c)])
        s["granted"] = _ints([0] * n)
        s["plan"] = _ints([-1] * (1 + 2 * n))
    else:
        s["plan"] = _ints([-1] * (1 + 2 * (pages // 2)))
    if c["kind"] in ("fork", "compact"):                      # the bookkeeping that a pass begins with
        s["began"] = [s[k].clone() for k in ("table", "len", "refs")]
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------

def _cached(s, table):
    """[slots, heads, tokens, dim] keys and values in fp32 of the pages that a table names (-1: any)."""
    c = s["case"]
    at = table.clamp(min=0).long()
    ex = torch.exp2(s["exps"][0][at].float())                                     # slots, pages, heads, blocks, 2
    k = _floats(s["k"][0][at]) * ex[..., 0, None, None, None, None]
    v = _floats(s["v"][0][at]) * ex[..., 1, None, None, None, None, None]
    join = lambda x: x.transpose(1, 2).reshape(x.shape[0], c["heads"], -1, c["dim"])  # noqa: E731
    return join(_k_rows(k, c)), join(_v_rows(v, c))


def _plain_attend(s):
    c = s["case"]
    n, h, g, d = c["slots"], c["heads"], c["group"], c["dim"]
    count = s["start"].diff()
    most = max(r for r, _ in _rows(c))
    i = torch.arange(most, device=DEV)
    there = i < count[:, None]                                                    # slots, rows
    row = (s["start"][:-1, None] + i).clamp(max=s["q"].shape[0] - 1).long()
    k, v = _cached(s, s["table"])
    q = s["q"][row].float().reshape(n, most, h, g, d).permute(0, 2, 3, 1, 4).reshape(n, h, g * most, d)
    scores = (q @ k.transpose(-1, -2)).reshape(n, h, g, most, -1) / math.sqrt(d)
    p = (s["len"] - count)[:, None, None] + i[:, None]                            # position of a row
    j = torch.arange(k.shape[2], device=DEV)
    seen = (j <= p) & (s["table"] >= 0).repeat_interleave(c["page"], 1)[:, None]
    if c["window"]:
        seen &= (j > p - c["window"]) | (j < c["sinks"])
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    scores.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = scores.sum(-1, keepdim=True)
    out = (scores.reshape(n, h, g * most, -1) @ v).reshape(n, h, g, most, d)
    out = torch.where(total > 0, out / total, 0.0).permute(0, 3, 1, 2, 4).reshape(n, most, h * g, d)
    s["out"][row[there]] = out[there].to(s["out"].dtype)
    return s["out"]


def _plain_store(s):
    c = s["case"]
    n, h, d, page = c["slots"], c["heads"], c["dim"], c["page"]
    count, end = s["start"].diff(), s["len"]
    begin = end - count
    blocks = max(r for r, _ in _rows(c)) // BLOCK + 2                             # that a slot's new tokens touch, at most
    b = begin[:, None] // BLOCK + torch.arange(blocks, device=DEV)                # slots, blocks
    pos = b[:, :, None] * BLOCK + torch.arange(BLOCK, device=DEV)                 # slots, blocks, 16
    fresh = (pos >= begin[:, None, None]) & (pos < end[:, None, None])
    older = (pos < begin[:, None, None]) & fresh.any(-1, keepdim=True)
    row = (s["start"][:-1, None, None] + pos - begin[:, None, None]).clamp(0, s["new_k"].shape[0] - 1).long()
    per = page // BLOCK
    here = s["table"].gather(1, (b // per).clamp(0, s["table"].shape[1] - 1).long()).clamp(min=0).long()
    touched = fresh.any(-1)
    slot, at = torch.nonzero(touched, as_tuple=True)
    where, sub = here[slot, at], (b % per)[slot, at].long()
    for which, pool, lay, unlay, new in ((0, s["k"][0], _k_lay, _k_rows, s["new_k"]), (1, s["v"][0], _v_lay, _v_rows, s["new_v"])):
        x = new[row[slot, at]].float().movedim(2, 1)                              # blocks, heads, 16, dim
        is_new, is_old = (m[slot, at][:, None, :, None] for m in (fresh, older))
        e = _exponent(torch.where(is_new, x, 0.0))
        old = unlay(pool[where, :, sub][:, :, None], c)                           # blocks, heads, 16, dim
        was = s["exps"][0][where, :, sub, which].int()
        e = torch.where(is_old.any(2)[..., 0], torch.maximum(e, was), e)
        again = _codes(_floats(old.contiguous()), e - was)
        keep = torch.where(is_old, again, torch.where(is_new, _codes(x, e), 0))
        pool[where, :, sub] = lay(keep, c)[:, :, 0]
        s["exps"][0][where, :, sub, which] = e.to(torch.int8)
    k, v = _cached(s, s["table"])
    j = (end[s["slots"].long()] - c["new"])[:, None] + torch.arange(c["new"], device=DEV)
    index = j.clamp(min=0).long()[:, None, :, None].expand(n, h, c["new"], d)
    most = torch.finfo(s["out_k"].dtype).max
    for x, to in ((k, s["out_k"]), (v, s["out_v"])):
        y = x[s["slots"].long()].gather(2, index).clamp(-most, most)
        to.copy_(torch.where((j >= 0)[:, None, :, None], y, 0.0))
    return s["out_k"], s["out_v"]


def _free_first(refs):
    """Indices of free pages, ascending, then the others."""
    return torch.argsort((refs != 0).to(torch.int8), stable=True)


def _move(s, pages_from, pages_to):
    for x in (s["k"], s["v"], s["exps"]):
        x[:, pages_to] = x[:, pages_from]


def _plain_fork(s):
    c = s["case"]
    n, page, wide = c["slots"], c["page"], s["table"].shape[1]
    source = s["from"].long()
    kept = source >= 0
    s["table"].copy_(torch.where(kept[:, None], s["table"][source.clamp(min=0)], -1))
    s["len"].copy_(torch.where(kept, s["len"][source.clamp(min=0)], 0))
    held = s["table"][s["table"] >= 0].long()
    s["refs"].copy_(torch.bincount(held, minlength=s["refs"].numel()))
    # room: a copy of the page that goes on being filled, for every slot but the last one that shares it, and new pages
    end = s["len"] + s["wanted"]
    wants = s["wanted"] > 0
    part = s["len"] // page
    open_page = s["table"].gather(1, part.clamp(max=wide - 1).long()[:, None])[:, 0]
    writes = wants & (s["len"] % page != 0)
    same = (open_page[:, None] == open_page) & writes[:, None] & writes
    before = (same & torch.ones(n, n, dtype=torch.bool, device=DEV).tril(-1)).sum(1)
    copies = writes & (s["refs"][open_page.clamp(min=0).long()] - before > 1)
    first = part + (s["len"] % page != 0) - copies.int()
    need = torch.where(wants, -(-end // page) - first, 0)
    upto = need.cumsum(0)
    fits = upto <= (s["refs"] == 0).sum()
    fits = (fits | ~wants).int().cumprod(0).bool()
    s["granted"].copy_(torch.where(fits, s["wanted"], 0))
    take = _free_first(s["refs"])
    j = torch.arange(wide, device=DEV)
    mine = fits[:, None] & wants[:, None] & (j >= first[:, None]) & (j < (first + need)[:, None])
    page_of = take[((upto - need)[:, None] + j - first[:, None]).clamp(0, take.numel() - 1)]
    old, copied = open_page.long(), copies & fits
    s["refs"].sub_(torch.bincount(old[copied], minlength=s["refs"].numel()))
    s["table"].copy_(torch.where(mine, page_of, s["table"]))
    s["refs"][page_of[mine]] = 1
    s["len"].copy_(torch.where(fits, end, s["len"]))
    pairs = torch.stack([old, s["table"].gather(1, part.clamp(max=wide - 1).long()[:, None])[:, 0].long()], 1)[copied]
    s["plan"][:1] = copied.sum()
    s["plan"][1:1 + 2 * pairs.shape[0]] = pairs.reshape(-1).int()
    _move(s, pairs[:, 0], pairs[:, 1])


def _plain_compact(s):
    used = s["refs"] > 0
    count = used.sum()
    i = torch.arange(used.numel(), device=DEV)
    source, to = torch.nonzero(used & (i >= count))[:, 0], torch.nonzero(~used & (i < count))[:, 0]
    goes = i.clone()
    goes[source] = to
    s["table"].copy_(torch.where(s["table"] >= 0, goes[s["table"].clamp(min=0).long()], -1))
    s["refs"][to] = s["refs"][source]
    s["refs"][source] = 0
    s["plan"][:1] = source.numel()
    s["plan"][1:1 + 2 * source.numel()] = torch.stack([source, to], 1).reshape(-1).int()
    _move(s, source, to)


# ---- a pass ----------------------------------------------------------------------------------------------------------------

def _cache(s):
    """The program's handle on its buffers, made once."""
    if "cache" not in s:
        from paper_2402_09398_amd import PagedCache
        c = s["case"]
        s["cache"] = PagedCache(c["slots"], s["refs"].numel(), c["page"], s["table"].shape[1], c["heads"], c["dim"], c["dtype"],
                                layers=c["layers"], q_per_kv=c["group"], sinks=c["sinks"], window=c["window"],
                                max_rows=s["q"].shape[0] if "q" in s else 0, device=DEV,
                                buffers={"k_codes": s["k"], "v_codes": s["v"], "exps": s["exps"], "table": s["table"],
                                         "length": s["len"], "refs": s["refs"]})
    return s["cache"]


def run(s):
    c = s["case"]
    kind = c["kind"]
    if kind in ("fork", "compact"):
        for name, value in zip(("table", "len", "refs"), s["began"]):
            s[name].copy_(value)
    if own:
        cache = _cache(s)
        if kind == "store":
            cache.append(0, s["new_k"], s["new_v"], s["start"])
            cache.read(0, s["slots"], -c["new"], s["out_k"], s["out_v"])
            return s["out_k"], s["out_v"]
        if kind == "attend":
            cache.attend(0, s["q"], s["out"], s["start"], c["new"])
            return s["out"]
        if kind == "fork":
            cache.select(s["from"])
            cache.reserve(s["wanted"], s["granted"], s["plan"])
            cache.copy(s["plan"], c["slots"])
        else:
            cache.compact(s["plan"])
            cache.copy(s["plan"], s["refs"].numel() // 2)
    elif kind == "store":
        return _plain_store(s)
    elif kind == "attend":
        return _plain_attend(s)
    elif kind == "fork":
        _plain_fork(s)
    else:
        _plain_compact(s)
    names = ("table", "len", "refs", "plan", "k", "v", "exps") + (("granted",) if kind == "fork" else ())
    return {name: s[name] for name in names}


# ---- in 64 bits -----------------------------------------------------------------------------------------------------------

def _value_of(code):
    """What an e4m3 code stands for: sign, four bits of exponent, three of mantissa."""
    code = code.long()
    e, m = (code >> 3) & 15, code & 7
    x = torch.where(e > 0, (8 + m).double() * torch.exp2((e - 10).double()), m.double() * 2.0 ** -9)
    x = torch.where((code & 127) == 127, math.nan, x)
    return torch.where(code >= 128, -x, x)


def _token(s, slot, name, which, pool):
    """[heads, tokens, dim] of a slot in float64, channel by channel from the description of a block."""
    c = s["case"]
    n = int(s["len"][slot])
    t, d = torch.arange(n, device=DEV)[:, None], torch.arange(c["dim"], device=DEV)
    page = s["table"][slot].long()[t // c["page"]].clamp(min=0)
    block, i = t % c["page"] // BLOCK, t % BLOCK
    if which == 0:
        got = pool[0][page, :, block, d // 64, d % 64 // 16, i, d % 16]
    else:
        got = pool[0][page, :, block, d // 64, i // 4, d % 16, d % 64 // 16, i % 4]
    e = s["exps"][0][page, :, block, which].double()
    return (_value_of(got) * torch.exp2(e)).permute(2, 0, 1)


def _nearest(x, e):
    """x to the nearest value of the form that a code with exponent e can have, ties to even."""
    y = x / torch.exp2(e)
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(y / step) * step * torch.exp2(e)


def exact(c, seed):
    if c["kind"] not in ("store", "attend"):
        return None                                           # whole numbers and bytes that move
    s = prepare(c, seed)
    rows, h, g, d = _rows(c), c["heads"], c["group"], c["dim"]
    if c["kind"] == "attend":
        cost = sum(_pairs(c, *r)[0] + r[0] * r[1] for r in rows) * h * g
        if cost > 6e10:
            return None
        out, at = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV), 0
        for slot, (new, length) in enumerate(rows):
            if not new:
                continue
            k, v = (_token(s, slot, c, w, s[x]) for w, x in ((0, "k"), (1, "v")))
            step = max(1, 400_000_000 // max(1, length * g))
            for a in range(0, new, step):
                b = min(new, a + step)
                p = torch.arange(length - new + a, length - new + b, device=DEV)[:, None]
                j = torch.arange(length, device=DEV)
                seen = j <= p
                if c["window"]:
                    seen = seen & ((p - j < c["window"]) | (j < c["sinks"]))
                for head in range(h):
                    q = s["q"][at + a:at + b, head * g:(head + 1) * g].double().transpose(0, 1)
                    x = torch.matmul(q, k[head].t().contiguous()) * d ** -0.5
                    x = torch.where(seen, x, -math.inf)
                    x = torch.exp(x - x.amax(-1, keepdim=True))
                    y = torch.matmul(x, v[head]) / x.sum(-1, keepdim=True)
                    out[at + a:at + b, head * g:(head + 1) * g] = y.transpose(0, 1)
            at += new
        return out
    got = []
    for which, pool, new in ((0, "k", "new_k"), (1, "v", "new_v")):
        out, at = torch.zeros(s["out_k"].shape, dtype=torch.float64, device=DEV), 0
        for slot, (fresh, length) in enumerate(rows):
            first = length - fresh
            x = _token(s, slot, c, which, s[pool])
            x[:, first:] = s[new][at:at + fresh].double().transpose(0, 1)
            pad = -length % BLOCK
            x = torch.cat([x, x.new_zeros(h, pad, d)], 1).reshape(h, -1, BLOCK, d)
            isnew = torch.zeros(length + pad, dtype=torch.bool, device=DEV)
            isnew[first:length] = True
            isnew = isnew.reshape(1, -1, BLOCK, 1)
            top = torch.where(isnew, x.abs(), 0.0).amax((-1, -2))
            e = torch.ceil(torch.log2(top.clamp(min=2.0 ** -80) / 448)).clamp(-40, 40)
            nb = (length + pad) // BLOCK
            per = c["page"] // BLOCK
            b = torch.arange(nb, device=DEV)
            was = s["exps"][0][s["table"][slot].long()[b // per].clamp(min=0), :, b % per, which].double().t()
            started = torch.arange(nb, device=DEV) * BLOCK < first
            e = torch.where(started, torch.maximum(e, was), e)
            e = torch.where(isnew.any(2)[..., 0], e, was)[..., None, None]
            x = _nearest(x, e).reshape(h, -1, d)[:, :length]
            count = min(length, c["new"])
            out[slot, :, c["new"] - count:] = x[:, length - count:]
            at += fresh
        got.append(out)
    return got
