"""Performance cases of what follows several continuations of a prompt: beams, or samples, over the compressed and the paged cache.

Three kinds of pass, each what a serving program does in one go:

* ``beam``: the next beams of every prompt from the logits of its beams: the best (beam, token) pairs by the sum of log-probabilities, with
  their parents, which are what a cache's ``select`` takes.
* ``states``: the compressed states of a layer follow their beams: row b becomes what row ``source[b]`` was, in place.
* ``prefix``: attention of every slot's newest tokens over a paged cache whose slots share pages: what they have in common is looked
  for once for all layers, and read once for all slots that share it.

Head shapes are those of Llama 2 7B / 13B (32 / 40 heads of 128), the Falcon shape (71 query heads of 64 on one key/value head) and
grouped heads as ``bench.py --q-per-kv`` makes them; queries and keys N(0, sigma^2) with sigma ~ U[0.5, 2] per head, values N(0, 1).
"""
from __future__ import annotations

import math

import torch

own = False

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 16


def _beam(groups, beams, vocab, dtype="f16", picks=0, pad=0, end=True, name=None):
    c = {} if name is None else {"name": name}
    c.update(kind="beam", groups=groups, beams=beams, vocab=vocab, dtype=dtype, picks=picks or beams, pad=pad, end=end)
    return c


def _states(batch, heads, dim, heavy, recent, rank, beams, dtype="f16", ended=False, name=None):
    c = {} if name is None else {"name": name}
    c.update(kind="states", batch=batch, heads=heads, dim=dim, heavy=heavy, recent=recent, rank=rank, beams=beams, dtype=dtype, ended=ended)
    return c


def _prefix(slots, heads, dim, page, prompt, rest, prompts=1, system=0, new=1, group=1, dtype="f16", sinks=0, window=0, layers=1, name=None):
    """`prompts` prompts of up to `prompt` tokens, all of them behind the same `system` ones, shared by slots / prompts slots each, of which
    each has up to `rest` tokens of its own, the `new` ones among them."""
    c = {} if name is None else {"name": name}
    c.update(kind="prefix", slots=slots, heads=heads, dim=dim, page=page, prompt=prompt, rest=rest, prompts=prompts, system=system,
             new=new, group=group, dtype=dtype, sinks=sinks, window=window, layers=layers)
    return c


def listed():
    return [
        # four beams of one request on Llama 2's vocabulary: latency
        _beam(1, 4, 32000, name="beam-32000-b1x4"),
        # eight beams of 16 requests, a vocabulary of odd size in rows that lie apart, twice as many candidates as beams
        _beam(16, 8, 50257, "f32", picks=16, pad=7, end=False, name="beam-50257-b16x8"),
        # a full batch on a large vocabulary
        _beam(64, 4, 128256, "bf16", name="beam-128256-b64x4"),
        # the compressed states of two requests' beams, one layer of the 7B model
        _states(8, 32, 128, 51, 51, 8, 4, name="states-7b-b8"),
        # the batch of the throughput runs, some requests at their end
        _states(64, 32, 128, 51, 51, 8, 4, ended=True, name="states-7b-b64"),
        # the 13B model at 10 % of 4096 tokens, rank 16, eight beams
        _states(32, 40, 128, 204, 204, 16, 8, name="states-13b-10pct-b32"),
        # four samples of one prompt on the 7B model, one layer: latency
        _prefix(4, 32, 128, 16, 1030, 40, name="samples-7b-b4"),
        # 64 beams of one long prompt, grouped query heads
        _prefix(64, 8, 128, 16, 8192, 300, group=4, dtype="bf16", layers=4, name="beams-gqa4-b64"),
        # four samples of each of 16 uneven prompts, all behind the same instructions
        _prefix(64, 8, 128, 32, 3500, 400, prompts=16, system=1000, group=8, layers=2, name="samples-gqa8-b16x4"),
        # questions of a few dozen tokens about one long document
        _prefix(32, 32, 128, 64, 16384, 500, new=24, dtype="bf16", layers=1, name="questions-7b-b32"),
        # one very long document, a token of every answer
        _prefix(24, 8, 128, 64, 131072, 1000, group=5, layers=1, name="document-gqa5-b24"),
        # Falcon's 71 query heads on one key/value head, first tokens and a window
        _prefix(64, 1, 64, 32, 8192, 300, group=71, sinks=4, window=2044, layers=4, name="beams-mqa71-window"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["beam", "beam", "states", "prefix", "prefix", "prefix"])
    if kind == "beam":
        dtype = rng.choice(["f32", "f16", "bf16"])
        beams = rng.choice([1, 2, 3, 4, 4, 5, 8, 16, rng.randint(17, 64)])
        vocab = _log(rng, 500, 130000)
        most = 64 * 4 * 128256 // (vocab * beams)
        return _beam(_log(rng, 1, max(1, min(128, most))), beams, vocab, dtype, picks=min(64, rng.choice([1, 1, 2]) * beams),
                     pad=rng.choice([0, 0, rng.randint(1, 63)]), end=rng.random() < 0.6)
    if kind == "states":
        heads, dim = rng.choice([32, 40, 12, 8, 1]), rng.choice([128, 128, 64])
        heavy, recent = _log(rng, 1, 204), _log(rng, 1, 204)
        room = 64 * 32 * 128 * 102 * 5 // (heads * dim * (heavy + recent))
        return _states(_log(rng, 2, max(2, min(192, room))), heads, dim, heavy, recent, rng.choice([4, 8, 8, 16, rng.randint(1, 64)]),
                       rng.choice([2, 3, 4, 4, 5, 8, 16]), rng.choice(["f16", "f16", "f32"]), rng.random() < 0.5)
    dim = rng.choice([128, 128, 64])
    group = rng.choice([1, 1, 2, 3, 4, 5, 8, 16, 71 if dim == 64 else 12])
    heads = 1 if group == 71 else max(1, rng.choice([32, 40, 12, 8]) // group)
    prompts = rng.choice([1, 1, 1, _log(rng, 2, 16)])
    slots = prompts * _log(rng, 2, 64 // prompts) if prompts < 32 else prompts
    sinks, window = rng.choice([(0, 0), (0, 0), (0, 0), (4, _log(rng, 64, 4096)), (0, _log(rng, 16, 4096)), (rng.randint(1, 70), _log(rng, 1, 700))])
    new = rng.choice([1, 1, 1, _log(rng, 2, 40)])
    most = min(131072, 32 * 32 * 128 * 16384 // (slots * heads * dim))
    prompt = _log(rng, 64, most // 2)
    system = rng.choice([0, 0, _log(rng, 16, most // 2)]) if prompts > 1 else 0
    return _prefix(slots, heads, dim, rng.choice([16, 16, 32, 64, 128]), prompt, new + _log(rng, 1, 600), prompts, system, new, group,
                   rng.choice(["f16", "bf16"]), sinks, window, rng.choice([1, 1, 2]))


# ---- sizes of a case, the same for every seed --------------------------------------------------------------------------

def _share(i, n):
    """Spread evenly over (0.1, 1], the last one 1."""
    return 1.0 if i == n - 1 else 0.1 + 0.9 * ((i + 1) * 0.6180339887 % 1.0)


def _slots(c):
    """(prompt it belongs to, tokens shared by all, tokens that its prompt's slots share, tokens of its own, new ones among them) of every slot."""
    got, each = [], c["slots"] // c["prompts"]
    for i in range(c["slots"]):
        p = min(i // each, c["prompts"] - 1)
        prompt = max(1, round(c["prompt"] * _share(p, c["prompts"])))
        rest = max(c["new"], round(c["rest"] * _share(i, c["slots"])))
        got.append((p, c["system"], prompt, rest, c["new"]))
    return got


def _parents(c):
    """What each batch row becomes a copy of: beams with uneven parents; with `ended`, every ninth request's rows become empty."""
    k, got = c["beams"], []
    for b in range(c["batch"]):
        first = b // k * k
        many = min(k, c["batch"] - first)
        at = b - first
        got.append(-1 if c["ended"] and b // k % 9 == 4 else first + (at // 2 + b // k) % many)
    return got


def _row_bytes(c):
    elem, C = (4 if c["dtype"] == "f32" else 2), c["heavy"] + c["recent"]
    kv = 2 * C * c["dim"] * elem
    return c["heads"] * (kv + C * (8 + 4 + 4 * c["rank"]) + 4 * c["rank"] * c["dim"] + 8 * c["rank"] + 8 + c["dim"] * elem + 4 * c["rank"])


def _seen(c, first, last):
    """Tokens that a row at one of the positions first .. last sees, as ranges."""
    w = c["window"]
    if not w or first < w:
        return [(0, last + 1)]
    lo = first - w + 1
    return [(0, min(c["sinks"], lo)), (lo, last + 1)]


def _pairs(c, first, last):
    w, s, n = c["window"], c["sinks"], 0
    for p in range(first, last + 1):
        lo = max(0, p + 1 - w) if w else 0
        n += p + 1 - lo + min(s, lo)
    return n


def _union(ranges):
    n, upto = 0, 0
    for a, b in sorted(ranges):
        n += max(0, b - max(a, upto))
        upto = max(upto, b)
    return n


def work(c):
    if c["kind"] == "beam":
        rows = c["groups"] * c["beams"]
        return {"bytes": rows * (c["vocab"] * (4 if c["dtype"] == "f32" else 2) + 5) + c["groups"] * c["picks"] * 13, "flops": 2 * rows * c["vocab"]}
    if c["kind"] == "states":
        to = [(b, f) for b, f in enumerate(_parents(c)) if f != b]
        one = _row_bytes(c)
        return {"bytes": one * (len({f for _, f in to if f >= 0}) + sum(f >= 0 for _, f in to)), "flops": 0}
    cut = lambda ranges, a, b: [(max(a, x), min(b, y)) for x, y in ranges if x < b and y > a]  # noqa: E731
    of_all, of_prompt, tokens, pairs, rows = [], {}, 0, 0, 0
    for p, system, prompt, rest, new in _slots(c):
        end = system + prompt + rest
        seen = _seen(c, end - new, end - 1)
        of_all += cut(seen, 0, system)
        of_prompt.setdefault(p, []).extend(cut(seen, system, system + prompt))
        tokens += _union(cut(seen, system + prompt, end))
        pairs += _pairs(c, end - new, end - 1)
        rows += new
    tokens += _union(of_all) + sum(_union(r) for r in of_prompt.values())
    tok = c["heads"] * c["dim"]
    return {"bytes": c["layers"] * (tokens * (2 * tok + c["heads"] * 2 / BLOCK) + 4 * rows * tok * c["group"]),
            "flops": c["layers"] * 4 * tok * c["group"] * pairs}


# ---- what a program has in hand -----------------------------------------------------------------------------------------

def _ints(values):
    return torch.tensor(values, dtype=torch.int32).to(DEV)


def _prepare_beam(c, g):
    rows, t = c["groups"] * c["beams"], TYPES[c["dtype"]]
    x = torch.randn(rows, c["vocab"] + c["pad"], generator=g, device=DEV) * 2.5
    likely = torch.randint(0, c["vocab"], (rows, 24), generator=g, device=DEV)
    x.scatter_add_(1, likely, 6 + 3 * torch.rand(rows, 24, generator=g, device=DEV))
    banned = torch.randint(0, c["vocab"], (rows, max(1, c["vocab"] // 100)), generator=g, device=DEV)
    x.scatter_(1, banned, -math.inf)                          # what a grammar does not allow
    s = {"logits": x.to(t)[:, :c["vocab"]], "score": -20 * torch.rand(rows, generator=g, device=DEV)}
    s["ended"] = (torch.rand(rows, generator=g, device=DEV) < 0.1) if c["end"] else None
    s["end_token"] = 2 if c["end"] else -1
    n = c["groups"] * c["picks"]
    s["parent"], s["token"] = _ints([0] * n), _ints([0] * n)
    s["next_score"] = torch.zeros(n, device=DEV)
    s["next_ended"] = torch.zeros(n, dtype=torch.bool, device=DEV)
    return s


def _prepare_states(c, g):
    B, H, D, C, R, t = c["batch"], c["heads"], c["dim"], c["heavy"] + c["recent"], c["rank"], TYPES[c["dtype"]]
    normal = lambda *shape: torch.randn(*shape, generator=g, device=DEV)  # noqa: E731
    full = torch.randint(C, 5000, (B, H), generator=g, device=DEV, dtype=torch.int32)
    s = {"k_cache": normal(B, H, C, D).to(t), "v_cache": normal(B, H, C, D).to(t), "acc": normal(B, H, C).double().abs(),
         "pos": torch.randint(0, 5000, (B, H, C), generator=g, device=DEV, dtype=torch.int32), "psi": normal(B, H, C, R).abs(),
         "H": normal(B, H, R, D), "z": normal(B, H, R).double().abs(), "n_seen": full,
         "pend_slot": torch.randint(-1, C, (B, H), generator=g, device=DEV, dtype=torch.int32), "pend_v": normal(B, H, D).to(t),
         "pend_psi": normal(B, H, R).abs()}
    return {"state": s, "source": _ints(_parents(c))}


def _floats(codes):
    return codes.view(torch.float8_e4m3fn).float()


def _exponent(x):
    """Of blocks [..., 16, dim]: the least e with every magnitude within 448 * 2^e, at least -40."""
    m, e = torch.frexp(x.abs().amax((-1, -2)))
    return torch.where(m > 0, e - 9 + (m > 0.875), -40).clamp(-40, 40)


def _codes(x, e):
    return torch.ldexp(x, -e[..., None, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _pool(c, pages, g):
    """A pool of pages full of tokens: codes of keys and values as the cache lays them out, and exponents [layer, page, head, block, 2]."""
    blocks, h = c["page"] // BLOCK, c["dim"] // 64
    sigma = 0.5 + 1.5 * torch.rand(c["heads"], generator=g, device=DEV)
    k = torch.empty(c["layers"], pages, c["heads"], blocks, h, 4, 16, 16, dtype=torch.uint8, device=DEV)
    v = torch.empty(c["layers"], pages, c["heads"], blocks, h, 4, 16, 4, 4, dtype=torch.uint8, device=DEV)
    e = torch.empty(c["layers"], pages, c["heads"], blocks, 2, dtype=torch.int8, device=DEV)
    for layer in range(c["layers"]):
        x = torch.randn(pages, c["heads"], blocks, BLOCK, c["dim"], generator=g, device=DEV) * sigma[:, None, None, None]
        e[layer, ..., 0] = ex = _exponent(x)
        k[layer] = _codes(x, ex).reshape(pages, c["heads"], blocks, 16, h, 4, 16).permute(0, 1, 2, 4, 5, 3, 6)
        x.normal_(generator=g)
        e[layer, ..., 1] = ex = _exponent(x)
        v[layer] = _codes(x, ex).reshape(pages, c["heads"], blocks, 4, 4, h, 4, 16).permute(0, 1, 2, 5, 3, 7, 6, 4)
    return k, v, e


def _prepare_prefix(c, g):
    slots, page = _slots(c), c["page"]
    length = [system + prompt + rest for _, system, prompt, rest, _ in slots]
    width = -(-max(length) // page)
    # a page is shared where all of its tokens are: by all, by a prompt's slots, or by none
    names, count = {}, 0
    table = torch.full((c["slots"], width), -1, dtype=torch.int32)
    refs = []
    for i, (p, system, prompt, rest, new) in enumerate(slots):
        seen = _seen(c, length[i] - new, length[i] - 1)
        row = []
        for j in range(-(-length[i] // page)):
            held = any(a < (j + 1) * page and b > j * page for a, b in seen)          # (a page that no row sees any more has been let go)
            key = ("all", j) if (j + 1) * page <= system else (p, j) if (j + 1) * page <= system + prompt else (p, i, j)
            if not held:
                row.append(-1)
                continue
            if key not in names:
                names[key] = count
                count += 1
                refs.append(0)
            refs[names[key]] += 1
            row.append(names[key])
        table[i, :len(row)] = torch.tensor(row, dtype=torch.int32)
    pages = count + count // 16 + 2
    to = torch.randperm(pages, generator=g, device=DEV)[:count].int()
    s = {"table": torch.where(table.to(DEV) >= 0, to[table.clamp(min=0).to(DEV).long()], -1), "len": _ints(length)}
    s["refs"] = torch.zeros(pages, dtype=torch.int32, device=DEV)
    s["refs"][to.long()] = _ints(refs)
    s["k"], s["v"], s["exps"] = _pool(c, pages, g)
    starts = [0]
    for *_, new in slots:
        starts.append(starts[-1] + new)
    s["start"] = _ints(starts)
    heads = c["heads"] * c["group"]
    sigma = 0.5 + 1.5 * torch.rand(heads, 1, generator=g, device=DEV)
    s["q"] = (torch.randn(c["layers"], starts[-1], heads, c["dim"], generator=g, device=DEV) * sigma).to(TYPES[c["dtype"]])
    s["out"] = torch.zeros_like(s["q"])
    return s


def prepare(c, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed * 7919 + 31)
    s = {"beam": _prepare_beam, "states": _prepare_states, "prefix": _prepare_prefix}[c["kind"]](c, g)
    s["case"] = c
    return s


# ---- plain forms ----------------------------------------------------------------------------------------------------------

def _plain_beam(s):
    c = s["case"]
    rows, vocab = c["groups"] * c["beams"], c["vocab"]
    x = s["logits"].double()                                  # a choice hangs on small differences of large sums
    top = x.amax(1, keepdim=True)
    x = x - top
    x = s["score"].double()[:, None] + (x - x.exp().sum(1, keepdim=True).log())
    x = torch.where(x.isnan(), -math.inf, x)
    if s["ended"] is not None:
        x.masked_fill_(s["ended"][:, None], -math.inf)
        x[:, s["end_token"]] = torch.where(s["ended"], s["score"].double(), x[:, s["end_token"]])
    best, at = torch.sort(x.reshape(c["groups"], -1), dim=1, descending=True, stable=True)
    best, at = best[:, :c["picks"]], at[:, :c["picks"]]
    there = best > -math.inf
    first = torch.arange(0, rows, c["beams"], device=DEV)[:, None]
    s["parent"].copy_(torch.where(there, first + at // vocab, -1).reshape(-1))
    s["token"].copy_(torch.where(there, at % vocab, -1).reshape(-1))
    s["next_score"].copy_(best.reshape(-1))
    s["next_ended"].copy_((s["token"] >= 0) & (s["token"] == s["end_token"]))


def _plain_states(s):
    source = s["source"].long()
    stays = torch.arange(source.numel(), device=DEV)
    kept = torch.where(source < 0, stays, source)
    for name, x in s["state"].items():
        empty = -1 if name in ("pos", "pend_slot") else 0
        now = x[kept]
        if name not in ("k_cache", "v_cache", "pend_v", "pend_psi"):
            now[source < 0] = empty
        x.copy_(now)


def _cached(s, layer):
    """[slots, heads, tokens, dim] keys and values in fp32 of the pages that the table names (-1: any)."""
    c = s["case"]
    at = s["table"].clamp(min=0).long()
    n, pages = at.shape
    ex = torch.exp2(s["exps"][layer][at].float())
    k = _floats(s["k"][layer][at]) * ex[..., 0, None, None, None, None]            # slots, pages, heads, blocks, h, 4, 16 tokens, 16
    k = k.permute(0, 2, 1, 3, 6, 4, 5, 7).reshape(n, c["heads"], -1, c["dim"])
    v = _floats(s["v"][layer][at]) * ex[..., 1, None, None, None, None, None]      # .., h, 4 x 4 tokens (first, last), 16, 4
    v = v.permute(0, 2, 1, 3, 5, 8, 4, 7, 6).reshape(n, c["heads"], -1, c["dim"])
    return k, v


def _plain_prefix(s):
    c = s["case"]
    n, h, g, d, new = c["slots"], c["heads"], c["group"], c["dim"], c["new"]
    p = (s["len"] - new)[:, None, None] + torch.arange(new, device=DEV)[:, None]
    for layer in range(c["layers"]):
        k, v = _cached(s, layer)
        q = s["q"][layer].float().reshape(n, new, h, g, d).permute(0, 2, 3, 1, 4).reshape(n, h, g * new, d)
        scores = (q @ k.transpose(-1, -2)).reshape(n, h, g, new, -1) / math.sqrt(d)
        j = torch.arange(k.shape[2], device=DEV)
        seen = (j <= p) & (s["table"] >= 0).repeat_interleave(c["page"], 1)[:, None]
        if c["window"]:
            seen &= (j > p - c["window"]) | (j < c["sinks"])
        scores.masked_fill_(~seen[:, None, None], -math.inf)
        scores.sub_(scores.amax(-1, keepdim=True)).exp_()
        total = scores.sum(-1, keepdim=True)
        out = (scores.reshape(n, h, g * new, -1) @ v).reshape(n, h, g, new, d) / total
        s["out"][layer].copy_(out.permute(0, 3, 1, 2, 4).reshape(n * new, h * g, d))


# ---- a pass ----------------------------------------------------------------------------------------------------------------

def _handle(s):
    """The program's handle on its buffers, made once."""
    if "handle" not in s:
        c = s["case"]
        if c["kind"] == "beam":
            from paper_2402_09398_amd import BeamSearch
            s["handle"] = BeamSearch(c["groups"], c["beams"], c["vocab"], c["dtype"], picks=c["picks"], end_token=s["end_token"], device=DEV)
        elif c["kind"] == "states":
            from paper_2402_09398_amd import binding
            d = binding.Desc()
            d.batch, d.heads, d.head_dim, d.n_heavy, d.n_recent, d.rank = c["batch"], c["heads"], c["dim"], c["heavy"], c["recent"], c["rank"]
            d.hidden, d.dtype = 512, binding.DTYPE_F32 if c["dtype"] == "f32" else binding.DTYPE_F16
            for name, x in s["state"].items():
                setattr(d, name, x.data_ptr())
            s["handle"] = d
        else:
            from paper_2402_09398_amd import PagedCache
            s["handle"] = PagedCache(c["slots"], s["refs"].numel(), c["page"], s["table"].shape[1], c["heads"], c["dim"], c["dtype"],
                                     layers=c["layers"], q_per_kv=c["group"], sinks=c["sinks"], window=c["window"],
                                     max_rows=s["q"].shape[1], shared=True, device=DEV,
                                     buffers={"k_codes": s["k"], "v_codes": s["v"], "exps": s["exps"], "table": s["table"],
                                              "length": s["len"], "refs": s["refs"]})
            s["plan"] = s["handle"].share_plan()
    return s["handle"]


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        handle = _handle(s)
        if kind == "beam":
            handle.select(s["logits"], s["score"], s["ended"], s["parent"], s["token"], s["next_score"], s["next_ended"])
        elif kind == "states":
            from paper_2402_09398_amd import lessdec_state_select
            lessdec_state_select(handle, s["source"])
        else:
            handle.share(s["start"], s["q"].shape[1], s["plan"])
            for layer in range(c["layers"]):
                handle.attend_shared(layer, s["q"][layer], s["out"][layer], s["start"], c["new"], s["plan"])
    elif kind == "beam":
        _plain_beam(s)
    elif kind == "states":
        _plain_states(s)
    else:
        _plain_prefix(s)
    if kind == "beam":
        return s["parent"], s["token"], s["next_score"], s["next_ended"]
    return s["state"] if kind == "states" else s["out"]


# ---- in 64 bits -----------------------------------------------------------------------------------------------------------

def _value_of(code):
    """What an e4m3 code stands for: sign, four bits of exponent, three of mantissa."""
    code = code.long()
    e, m = (code >> 3) & 15, code & 7
    x = torch.where(e > 0, (8 + m).double() * torch.exp2((e - 10).double()), m.double() * 2.0 ** -9)
    return torch.where(code >= 128, -x, x)


def _exact_beam(c, s):
    scores = torch.full((c["groups"], c["picks"]), -math.inf, dtype=torch.float64, device=DEV)
    ended = s["ended"].tolist() if s["ended"] is not None else [False] * s["score"].numel()
    for group in range(c["groups"]):
        got = []
        for row in range(group * c["beams"], (group + 1) * c["beams"]):
            if ended[row]:
                got.append(s["score"][row:row + 1].double())
            else:
                x = s["logits"][row].double()
                got.append(s["score"][row].double() + x - torch.logsumexp(x, 0))
        best = torch.cat(got)
        best = torch.sort(best[best > -math.inf], descending=True)[0][:c["picks"]]
        scores[group, :best.numel()] = best
    return None, None, scores.reshape(-1), None


def _exact_states(c, s):
    got = {}
    for name, x in s["state"].items():
        got[name] = None
        if x.is_floating_point():
            old = x.double()
            rows = [old[b if f < 0 and name in ("k_cache", "v_cache", "pend_v", "pend_psi") else f] for b, f in enumerate(_parents(c))]
            got[name] = torch.stack([torch.zeros_like(r) if f < 0 and name in ("acc", "psi", "H", "z") else r for r, f in zip(rows, _parents(c))])
    return got


def exact(c, seed):
    if c["kind"] == "prefix" and c["layers"] * sum(_pairs(c, sum(x[1:4]) - x[4], sum(x[1:4]) - 1) for x in _slots(c)) * c["heads"] * c["group"] > 6e10:
        return None
    s = prepare(c, seed)
    if c["kind"] == "beam":
        return _exact_beam(c, s)
    if c["kind"] == "states":
        return _exact_states(c, s)
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEV)
    d, g, at = torch.arange(c["dim"], device=DEV), c["group"], 0
    for slot, (_, system, prompt, rest, new) in enumerate(_slots(c)):
        n = system + prompt + rest
        t = torch.arange(n, device=DEV)[:, None]
        held = s["table"][slot].long()[t[:, 0] // c["page"]]
        page, block, i = held[:, None].clamp(min=0), t % c["page"] // BLOCK, t % BLOCK
        p, j = torch.arange(n - new, n, device=DEV)[:, None], t[:, 0]
        seen = (j <= p) & (held >= 0)
        if c["window"]:
            seen = seen & ((p - j < c["window"]) | (j < c["sinks"]))
        for layer in range(c["layers"]):
            k = _value_of(s["k"][layer][page, :, block, d // 64, d % 64 // 16, i, d % 16])
            v = _value_of(s["v"][layer][page, :, block, d // 64, i // 4, d % 16, d % 64 // 16, i % 4])
            e = torch.exp2(s["exps"][layer][page, :, block].double())                       # tokens, 1, heads, 2
            for head in range(c["heads"]):
                q = s["q"][layer][at:at + new, head * g:(head + 1) * g].double().transpose(0, 1)
                x = torch.matmul(q, (k[:, :, head] * e[:, :, head, 0]).t().contiguous()) * c["dim"] ** -0.5
                x = torch.where(seen, x, -math.inf)
                x = torch.exp(x - x.amax(-1, keepdim=True))
                y = torch.matmul(x, v[:, :, head] * e[:, :, head, 1]) / x.sum(-1, keepdim=True)
                out[layer, at:at + new, head * g:(head + 1) * g] = y.transpose(0, 1)
        at += new
    return out
