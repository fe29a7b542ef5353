"""More operators of the paged cache of token sequences, as cases that can be timed and compared.

The cache holds K and V rows of sequences in pages that a table assigns, as bf16 or as 8-bit codes with one scale for each row.  Around it a
server of such a model does five more things:

  kind "rotate"  Q and K of new tokens are turned by their positions (time, height, width, or one axis for text), K and V join the cache
       "tree"    drafted tokens that form a tree attend: each sees everything before the draft, its ancestors and itself
       "accept"  the rows of a draft's accepted tokens move to the places behind what was there before, in all layers
       "weigh"   what attention each cached entry has got from the new tokens is added to its sum
       "evict"   of every sequence and kv head the entries with the largest sums stay, moved to other pages, beside the first and last ones

A case names the cache (`store`, `d`, `kv_heads`, `page`, `layers`), the batch (`seqs` sequences of up to `length` entries, `new` of them
new; `ragged`: lengths spread down to two fifths of that, new tokens likewise) and what its kind needs: `rows` the type of Q, K and V;
`axes` of the positions, `pairs` of dimensions that are turned, `adjacent` for pairs of neighbouring dimensions, `far` the range of the
positions; `window` and `sinks` of the mask of "weigh", `decay` of its sums; `keep`, `sinks` and `recent` of "evict"; `keep` accepted tokens.

The pool is laid out K rows, V rows, then for codes K scales, V scales, each [layer][page][kv head][row of the page].
"""
import math
import random

import torch

own = False

FIELDS = ("name", "kind", "store", "rows", "d", "heads", "kv_heads", "seqs", "new", "length", "ragged", "page", "layers", "axes", "pairs",
          "adjacent", "far", "window", "sinks", "decay", "keep", "recent")


def _case(*values):
    return dict(zip(FIELDS, values))


def listed():
    return [
        # one new token for each of 8 sequences, time, height and width: what a generated token costs ahead of its attention
        _case("rotate_tokens", "rotate", "q8", "bf16", 128, 32, 8, 8, 1, 1024, True, 64, 2, 3, 64, False, 100000, 0, 0, 1.0, 0, 0),
        # a 64 x 64 token map of two images, 16 heads, rows as they are
        _case("rotate_map", "rotate", "bf16", "bf16", 128, 16, 16, 2, 4096, 10521, False, 128, 2, 3, 64, False, 4096, 0, 0, 1.0, 0, 0),
        # rows in single precision, small heads of which three quarters turn, neighbouring dimensions, odd lengths, far positions
        _case("rotate_odd", "rotate", "q8", "f32", 64, 12, 4, 7, 333, 1999, True, 16, 2, 2, 24, True, 1 << 20, 0, 0, 1.0, 0, 0),
        # one user's draft of 8 tokens behind a caption and a past answer: latency
        _case("tree_one", "tree", "q8", "bf16", 128, 32, 8, 1, 8, 1999, False, 64, 2, 0, 0, False, 0, 0, 0, 1.0, 0, 0),
        # drafts of 64 tokens of 16 sequences of up to 10 521 entries: a serving step
        _case("tree_batch", "tree", "q8", "bf16", 128, 32, 8, 16, 64, 10521, True, 64, 2, 0, 0, False, 0, 0, 0, 1.0, 0, 0),
        # drafts of odd sizes behind short pasts, three heads to a kv head, small heads, rows as they are
        _case("tree_odd", "tree", "bf16", "bf16", 64, 12, 4, 24, 29, 777, True, 16, 2, 0, 0, False, 0, 0, 0, 1.0, 0, 0),
        # up to 8 of 64 drafted tokens of 32 sequences accepted, a model of 32 layers
        _case("accept_batch", "accept", "q8", "bf16", 128, 8, 8, 32, 64, 1024, True, 64, 32, 0, 0, False, 0, 0, 0, 1.0, 8, 0),
        # one user's draft: 3 of 8, small heads, rows as they are
        _case("accept_one", "accept", "bf16", "bf16", 64, 4, 4, 1, 8, 777, False, 16, 16, 0, 0, False, 0, 0, 0, 1.0, 3, 0),
        # the sums of 32 sequences of up to 10 521 entries behind every generated token
        _case("weigh_tokens", "weigh", "q8", "bf16", 128, 32, 8, 32, 1, 10521, True, 64, 2, 0, 0, False, 0, 0, 0, 1.0, 0, 0),
        # those of a chunk of 2 048 prompt tokens of four sequences behind 6 144 cached ones, old ones fading
        _case("weigh_prompt", "weigh", "q8", "bf16", 128, 32, 8, 4, 2048, 8192, False, 64, 2, 0, 0, False, 0, 0, 0, 0.95, 0, 0),
        # eight sequences as long as a 1024 x 1024 image's maps (10 521 tokens) down to a tenth of that
        _case("evict_batch", "evict", "q8", "bf16", 128, 8, 8, 8, 1, 10521, False, 64, 2, 0, 0, False, 0, 0, 4, 1.0, 1052, 64),
        # one as long as a 4K-class image's (170 521), 16 heads, rows as they are, a tenth stays
        _case("evict_long", "evict", "bf16", "bf16", 128, 16, 16, 1, 1, 170521, False, 128, 2, 0, 0, False, 0, 0, 4, 1.0, 17052, 1024),
    ]


def _spread(n, k):
    """n for k = 0, else between two fifths of it and all of it, evenly over k."""
    return max(1, round(n * (1.0 - 0.6 * ((k * 0.6180339887498949) % 1.0))))


def _new(case):
    return [_spread(case["new"], b) if case["ragged"] else case["new"] for b in range(case["seqs"])]


def _lengths(case):
    return [max(_spread(case["length"], b) if case["ragged"] else case["length"], n) for b, n in enumerate(_new(case))]


def _accepted(case):
    """How many tokens of each draft stay: never all of them, and none of a draft of one."""
    return [min(_spread(case["keep"], b), n - 1) if case["keep"] else 0 for b, n in enumerate(_new(case))]


def _kept(case):
    return [min(_spread(case["keep"], b) if case["ragged"] else case["keep"], l) for b, l in enumerate(_lengths(case))]


def _visible(case):
    """Of "weigh": (query, key) pairs that a head's mask leaves, and cached rows that some query sees."""
    pairs = rows = 0
    w, sinks = case["window"], case["sinks"]
    for n, length in zip(_new(case), _lengths(case)):
        first = length - n
        lo = max(0, first - w + 1) if w else 0
        rows += length - lo + min(sinks if w else 0, lo)
        for p in range(first, length):
            start = max(0, p - w + 1) if w else 0
            pairs += p + 1 - start + min(sinks if w else 0, start)
    return pairs, rows


def draw(rng):
    """One more case: any cache, batch and operator, from one token to chunks of thousands, odd sizes among them."""
    def log(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    while True:
        kind = rng.choice(["rotate", "rotate", "tree", "tree", "tree", "accept", "weigh", "weigh", "weigh", "evict", "evict"])
        store, d = rng.choice(["q8", "q8", "bf16"]), rng.choice([64, 128, 128])
        kv_heads, group = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([1, 1, 2, 3, 4, 8])
        length = log(1, 170000 if kind == "evict" else 40000)
        new = {"tree": log(1, min(length, 96)), "accept": log(1, min(length, 96)), "evict": 1,
               "weigh": 1 if rng.random() < 0.4 else log(1, min(length, 4096))}.get(kind, log(1, min(length, 4096)))
        window = log(16, 4096) if kind == "weigh" and rng.random() < 0.3 else 0
        keep = {"accept": log(1, 16), "evict": log(1, length)}.get(kind, 0)
        case = {"kind": kind, "store": store, "rows": rng.choice(["bf16", "bf16", "f32"]) if kind == "rotate" else "bf16", "d": d,
                "heads": kv_heads * (1 if kind in ("accept", "evict") else group), "kv_heads": kv_heads, "seqs": log(1, 64), "new": new,
                "length": length, "ragged": rng.random() < 0.7, "page": rng.choice([16, 32, 64, 64, 128]),
                "layers": log(1, 32) if kind == "accept" else 2, "axes": rng.choice([1, 2, 3, 4]) if kind == "rotate" else 0,
                "pairs": rng.choice([d // 2, d // 2, 24, 16, 8]) if kind == "rotate" else 0, "adjacent": kind == "rotate" and rng.random() < 0.4,
                "far": log(16, 1 << 22) if kind == "rotate" else 0, "window": window,
                "sinks": rng.choice([0, 1, 4, 16]) if window or kind == "evict" else 0,
                "decay": rng.choice([1.0, 0.95, 0.5]) if kind == "weigh" else 1.0, "keep": keep,
                "recent": log(1, keep) if kind == "evict" and rng.random() < 0.7 else 0}
        w = work(case)
        scores = case["seqs"] * case["heads"] * max(_new(case)) * max(_lengths(case)) if kind in ("tree", "weigh") else 0
        held = 2 * case["layers"] * case["seqs"] * max(_lengths(case)) * kv_heads * d * (4 if kind in ("tree", "weigh") else 2)
        if w["flops"] <= 2.8e11 and w["bytes"] <= 0.4e9 and w["bytes"] > 0 and scores <= 2.0e9 and held <= 8.0e9:
            return case


# ---- inputs -----------------------------------------------------------------------------------------------------------------------
def _generator(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 0x9E3779B1 + k * 0x85EBCA6B + 54321) & 0x7FFFFFFFFFFFFFFF)
    return g


def _offset(case, seed, what):
    """K rows of a head share an offset."""
    return 0.5 * torch.randn(1, case["kv_heads"], case["d"], generator=_generator(seed, 10 + what), device="cuda")


def _rows(case, seed, n, what):
    """[n, kv heads, d] K (what 0) or V rows: every 512th K row is a sink with four times the length."""
    x = torch.randn(n, case["kv_heads"], case["d"], generator=_generator(seed, what), device="cuda")
    if what == 0:
        x += _offset(case, seed, 0)
        x[::512] *= 4.0
    return x


def _row_type(case):
    return torch.float32 if case["rows"] == "f32" else torch.bfloat16


def _logical(case, seed, what):
    """The cached rows of all sequences, one behind the other: (codes or bf16 rows, scales or None)."""
    x = _rows(case, seed, sum(_lengths(case)), what)
    if case["store"] == "bf16":
        return x.bfloat16(), None
    s = x.abs().amax(-1) / torch.full((), 127.0, device="cuda")
    x /= s.unsqueeze(-1)
    return x.round_().to(torch.int8), s


def _queries(case, seed):
    return torch.randn(sum(_new(case)), case["heads"], case["d"], generator=_generator(seed, 2), device="cuda").to(_row_type(case))


def _starts(counts):
    return torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32, device="cuda")


def _positions(case, seed):
    """[axes, tokens]: a place in time somewhere in the range, and the token's place in rows of 16 from there on (more axes: anything)."""
    g, n = _generator(seed, 4), sum(_new(case))
    base = torch.randint(0, case["far"], (case["axes"], 1), generator=g, device="cuda")
    t = torch.arange(n, device="cuda")
    steps = torch.stack([t // 256, t // 16 % 16, t % 16, torch.randint(0, case["far"], (n,), generator=g, device="cuda")])
    return (base + (steps[2:3] if case["axes"] == 1 else steps[:case["axes"]])).to(torch.int32)


def _sections(case):
    """Pairs of each axis: as even as they come, the first axis with what is left."""
    each = case["pairs"] // case["axes"]
    return [case["pairs"] - each * (case["axes"] - 1)] + [each] * (case["axes"] - 1)


def _ancestors(case, seed):
    """For every drafted token the numbers of the draft's tokens that it sees: itself and its ancestors."""
    r, out = random.Random(seed * 7919 + 17), []
    for n in _new(case):
        sees = []
        for i in range(n):
            parent = r.randint(max(-1, i - 12), i - 1)
            sees.append((sees[parent] if parent >= 0 else []) + [i])
        out.append(sees)
    return out


def _bits(case, seed):
    """[tokens, words] int32: bit j of a token's words says that it sees token j of its draft."""
    words = -(-max(_new(case)) // 32)
    out = []
    for sees in _ancestors(case, seed):
        for js in sees:
            row = [0] * words
            for j in js:
                row[j // 32] |= 1 << (j % 32)
            out.append([w - (1 << 32) if w >= 1 << 31 else w for w in row])
    return torch.tensor(out, dtype=torch.int32, device="cuda")


def _paths(case, seed):
    """Numbers of the accepted tokens in their draft, ascending, none at the draft's first place: all of them move."""
    r = random.Random(seed * 7919 + 23)
    return [sorted(r.sample(range(1, n), k)) for n, k in zip(_new(case), _accepted(case))]


def _lse(case, seed):
    """Log-sum-exps as attention leaves them: those of normal rows, but for what one row differs from the next."""
    q = _queries(case, seed).float()
    group, d = case["heads"] // case["kv_heads"], case["d"]
    y = (q * _offset(case, seed, 0).repeat_interleave(group, 1)).sum(-1) / math.sqrt(d)
    seen = torch.cat([torch.arange(l - n, l, device="cuda") + 1.0 for n, l in zip(_new(case), _lengths(case))])
    if case["window"]:
        seen = seen.clamp(max=case["window"] + case["sinks"])
    return seen.log()[:, None] + y + q.square().sum(-1) / (2 * d) + 0.1 * torch.randn(y.shape, generator=_generator(seed, 5), device="cuda")


def _weights(case, seed, n):
    """[n, kv heads] sums of attention weights: a few heavy ones, some that nobody has looked at, and some equal ones."""
    g = _generator(seed, 6)
    w = torch.exp(2.0 * torch.randn(n, case["kv_heads"], generator=g, device="cuda") - 4.0)
    u = torch.rand(w.shape, generator=g, device="cuda")
    w = torch.where(u < 0.1, (w * 64).round() / 64, w)
    return torch.where(u > 0.97, torch.zeros_like(w), w)


def _region_bytes(case, pages):
    """Bytes of the K rows (or V rows) and of the K scales (or V scales)."""
    rows = case["layers"] * pages * case["kv_heads"] * case["page"]
    return rows * case["d"] * (1 if case["store"] == "q8" else 2), rows * 4 if case["store"] == "q8" else 0


def _table(case, order, need):
    table = torch.full((case["seqs"], max(max(need), 1)), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(need):
        table[b, :n] = order[sum(need[:b]): sum(need[: b + 1])]
    return table


def prepare(case, seed):
    new, lengths, page, layer = _new(case), _lengths(case), case["page"], case["layers"] - 1
    need = [-(-l // page) for l in lengths]
    need_to = [-(-k // page) for k in _kept(case)] if case["kind"] == "evict" else [0] * case["seqs"]
    pages = sum(need) + sum(need_to) + 3
    order = torch.randperm(pages, generator=_generator(seed, 3), device="cuda").to(torch.int32)      # pages were handed out in no order
    table = _table(case, order, need)
    rows_bytes, scale_bytes = _region_bytes(case, pages)
    pool = torch.zeros(2 * rows_bytes + 2 * scale_bytes, dtype=torch.uint8, device="cuda")
    shape = (case["layers"], pages, case["kv_heads"], page)
    dt = torch.int8 if case["store"] == "q8" else torch.bfloat16
    s = {"case": case, "layer": layer, "pool": pool, "table": table, "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"),
         "starts": _starts(new), "max_new": max(new), "max_length": max(lengths), "tokens": sum(new)}
    for i, name in enumerate(("K", "V")):
        s[name + "_rows"] = pool[i * rows_bytes: (i + 1) * rows_bytes].view(dt).view(*shape, case["d"])
        at = 2 * rows_bytes + i * scale_bytes
        s[name + "_scales"] = pool[at: at + scale_bytes].view(torch.float32).view(shape) if scale_bytes else None
    pos = torch.cat([torch.arange(l, device="cuda") for l in lengths])
    seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), s["lengths"].long())
    at, row = table[seq, pos // page].long(), pos % page
    if case["kind"] != "rotate":
        for i, name in enumerate(("K", "V")):
            codes, scales = _logical(case, seed, i)
            for l in range(case["layers"]) if case["kind"] == "accept" else [layer]:
                s[name + "_rows"][l, at, :, row] = codes
                if scales is not None:
                    s[name + "_scales"][l, at, :, row] = scales
    if case["kind"] == "rotate":
        s["Q"] = _queries(case, seed)
        s["K"], s["V"] = (_rows(case, seed, sum(new), i).to(_row_type(case)) for i in (0, 1))
        s["positions"] = _positions(case, seed)
        s["Q_out"] = torch.empty(s["Q"].shape, dtype=torch.bfloat16, device="cuda")
        shape = (sum(new), case["kv_heads"], case["d"])
        s["K_out"], s["V_out"] = (torch.empty(shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    elif case["kind"] == "tree":
        s["Q"], s["tree"] = _queries(case, seed), _bits(case, seed)
        s["O"], s["lse"] = torch.empty_like(s["Q"]), torch.empty(s["Q"].shape[:2], device="cuda")
    elif case["kind"] == "accept":
        paths = _paths(case, seed)
        most = max(1, max(len(p) for p in paths))
        s["path"] = torch.tensor([p + [-1] * (most - len(p)) for p in paths], dtype=torch.int32, device="cuda")
        s["counts"] = torch.tensor([len(p) for p in paths], dtype=torch.int32, device="cuda")
    elif case["kind"] == "weigh":
        s["Q"], s["lse"] = _queries(case, seed), _lse(case, seed)
    if case["kind"] in ("weigh", "evict"):
        s["weights"] = torch.zeros(pages, case["kv_heads"], page, device="cuda")
        s["weights"][at, :, row] = _weights(case, seed, sum(lengths))
    if case["kind"] == "evict":
        s["to"] = _table(case, order[sum(need):], need_to)
        s["keep"] = torch.tensor(_kept(case), dtype=torch.int32, device="cuda")
        s["kept"] = torch.full((case["seqs"], case["kv_heads"], max(_kept(case))), -1, dtype=torch.int32, device="cuda")
    if own:
        from paper_2505_19602_b200 import binding

        s["kv"] = binding.PagedKV(case["layers"], pages, case["kv_heads"], case["d"], store=case["store"], page_tokens=page, pool=pool)
        s["batch"] = binding.PagedBatch(table, s["lengths"], s["starts"], s["tokens"], s["max_new"], s["max_length"])
        if case["kind"] == "rotate":
            s["rotary"] = binding.Rotary(_sections(case), theta=10000.0, adjacent=case["adjacent"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if own:
        kv, layer, batch = s["kv"], s["layer"], s["batch"]
        if case["kind"] == "rotate":
            kv.scalekv_paged_write_rotated(layer, batch, s["Q"], s["K"], s["V"], s["rotary"], s["positions"], s["Q_out"])
            if case["store"] == "q8":
                kv.scalekv_paged_read(layer, batch, s["K_out"], s["V_out"])
        elif case["kind"] == "tree":
            kv.scalekv_paged_attend_tree(layer, batch, s["Q"], s["tree"], s["O"], lse=s["lse"])
        elif case["kind"] == "accept":
            kv.scalekv_paged_accept(batch, s["path"], s["counts"])
        elif case["kind"] == "weigh":
            kv.scalekv_paged_weigh(layer, batch, s["Q"], s["lse"], s["weights"], window=case["window"], n_sink=case["sinks"], decay=case["decay"], fade_hidden=True)
        else:
            kv.scalekv_paged_evict(layer, batch, s["to"], s["keep"], s["weights"], n_sink=case["sinks"], n_recent=case["recent"], kept=s["kept"])
    else:
        {"rotate": _rotate_plain, "tree": _tree_plain, "accept": _accept_plain, "weigh": _weigh_plain, "evict": _evict_plain}[case["kind"]](s)
    rows = {k: s[k] for k in ("K_rows", "V_rows", "K_scales", "V_scales") if s[k] is not None}
    if case["kind"] == "rotate":
        if case["store"] == "bf16":
            return {"Q": s["Q_out"], **rows}
        return {"Q": s["Q_out"], "K": s["K_out"], "V": s["V_out"], "K_scales": s["K_scales"], "V_scales": s["V_scales"]}
    if case["kind"] == "tree":
        return {"O": s["O"], "lse": s["lse"]}
    if case["kind"] == "accept":
        return rows
    if case["kind"] == "weigh":
        return {"weights": s["weights"]}
    return {"kept": s["kept"], "weights": s["weights"], **rows}


def _tokens(s):
    """Sequence and place among its new tokens of every new token."""
    t = torch.arange(s["tokens"], device="cuda", dtype=torch.int32)
    seq = torch.searchsorted(s["starts"], t, right=True) - 1
    return seq, t - s["starts"][seq]


def _where(s):
    """Page and row of every new token."""
    seq, i = _tokens(s)
    n = s["starts"][seq + 1] - s["starts"][seq]
    pos = (s["lengths"][seq] - n + i).long()
    return s["table"][seq, pos // s["case"]["page"]].long(), pos % s["case"]["page"]


def _write_plain(s, name, x):
    at, row = _where(s)
    if s["case"]["store"] == "bf16":
        s[name + "_rows"][s["layer"], at, :, row] = x.bfloat16()
        return
    a = x.abs().amax(-1)
    scale = a / torch.full_like(a, 127.0)
    codes = torch.where(scale.unsqueeze(-1) > 0, x / scale.unsqueeze(-1), torch.zeros_like(x)).round().clamp(-127, 127)
    s[name + "_rows"][s["layer"], at, :, row] = codes.to(torch.int8)
    s[name + "_scales"][s["layer"], at, :, row] = scale
    s[name + "_out"].copy_(s[name + "_rows"][s["layer"], at, :, row].float() * s[name + "_scales"][s["layer"], at, :, row].unsqueeze(-1))


def _pairs(case, x):
    """The turning dimensions of x as (first of each pair, second of each pair), and the dimensions that stay."""
    n = case["pairs"]
    if case["adjacent"]:
        return x[..., 0: 2 * n: 2], x[..., 1: 2 * n: 2], x[..., 2 * n:]
    return x[..., :n], x[..., n: 2 * n], x[..., 2 * n:]


def _joined(case, a, b, rest):
    turned = torch.stack((a, b), -1).flatten(-2) if case["adjacent"] else torch.cat((a, b), -1)
    return torch.cat((turned, rest), -1)


def _rotate_plain(s):
    case = s["case"]
    i = torch.arange(case["pairs"], device="cuda", dtype=torch.float64)
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"), torch.tensor(_sections(case), device="cuda"))
    angle = s["positions"].double()[axis].T * torch.pow(10000.0, -i / case["pairs"])      # [tokens, pairs]
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def turned(x):
        a, b, rest = _pairs(case, x.float())
        return _joined(case, a * cos - b * sin, a * sin + b * cos, rest)

    s["Q_out"].copy_(turned(s["Q"]))
    _write_plain(s, "K", turned(s["K"]))
    _write_plain(s, "V", s["V"].float())


def _gather_plain(s, name):
    """[sequences, kv heads, positions, d] in 32 bits, the table's holes from page 0 (no query sees them)."""
    table = s["table"].clamp(min=0).long()
    x = s[name + "_rows"][s["layer"]][table].float()
    if s["case"]["store"] == "q8":
        x = x * s[name + "_scales"][s["layer"]][table].unsqueeze(-1)
    return x.transpose(1, 2).flatten(2, 3)


def _products(s):
    """[sequences, kv heads, group, new tokens, positions]: scaled products of queries and keys; and which new tokens there are."""
    case = s["case"]
    B, H, G, N = case["seqs"], case["kv_heads"], case["heads"] // case["kv_heads"], s["max_new"]
    n = s["starts"][1:] - s["starts"][:-1]
    i = torch.arange(N, device="cuda", dtype=torch.int32)
    token = (s["starts"][:-1, None] + i).clamp(max=s["tokens"] - 1).long()
    Q = s["Q"][token].float().view(B, N, H, G, case["d"]).permute(0, 2, 3, 1, 4).reshape(B, H, G * N, case["d"])
    y = torch.matmul(Q, _gather_plain(s, "K").transpose(2, 3)).view(B, H, G, N, -1).mul_(1.0 / math.sqrt(case["d"]))
    return y, token, i < n[:, None]


def _tree_plain(s):
    case = s["case"]
    B, H, G, N = case["seqs"], case["kv_heads"], case["heads"] // case["kv_heads"], s["max_new"]
    y, token, _ = _products(s)
    n = s["starts"][1:] - s["starts"][:-1]
    j = torch.arange(y.shape[-1], device="cuda", dtype=torch.int32)
    k = j - (s["lengths"] - n)[:, None]                                                # a position's number in the draft
    word = (k // 32).clamp(0, s["tree"].shape[1] - 1).long()
    bits = torch.gather(s["tree"][token], 2, word[:, None].expand(-1, N, -1))
    seen = (k < 0)[:, None] | (((bits >> (k % 32)[:, None]) & 1) > 0) & (j < s["lengths"][:, None])[:, None]
    y.masked_fill_(~seen[:, None, None], -math.inf)
    top = y.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    y.sub_(top).exp_()
    total = y.sum(-1, keepdim=True)
    lse = (top + total.log()).view(B, H, G, N)
    O = torch.matmul(y.view(B, H, G * N, -1), _gather_plain(s, "V")).view(B, H, G, N, -1)
    O = torch.where(total > 0, O / total, torch.zeros_like(O))
    seq, place = _tokens(s)
    s["O"].copy_(O.permute(0, 3, 1, 2, 4).reshape(B, N, H * G, case["d"])[seq, place.long()])
    s["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(B, N, H * G)[seq, place.long()])


def _accept_plain(s):
    page = s["case"]["page"]
    i = torch.arange(s["path"].shape[1], device="cuda", dtype=torch.int32)
    seq, i = torch.nonzero(i < s["counts"][:, None], as_tuple=True)
    first = s["lengths"] - (s["starts"][1:] - s["starts"][:-1])
    src, dst = (first[seq] + s["path"][seq, i]).long(), first[seq].long() + i
    at, row, to, to_row = s["table"][seq, src // page].long(), src % page, s["table"][seq, dst // page].long(), dst % page
    rows = [s[k] for k in ("K_rows", "V_rows", "K_scales", "V_scales") if s[k] is not None]
    moved = [x[:, at, :, row] for x in rows]
    [x.index_put_((torch.arange(x.shape[0], device="cuda")[None, :, None], to[:, None, None], torch.arange(x.shape[2], device="cuda"), to_row[:, None, None]), y)
     for x, y in zip(rows, moved)]


def _entries(s):
    """Sequence, position, page and row of every cached entry."""
    j = torch.arange(s["max_length"], device="cuda", dtype=torch.int32)
    seq, pos = torch.nonzero(j < s["lengths"][:, None], as_tuple=True)
    return seq, pos, s["table"][seq, pos // s["case"]["page"]].long(), pos % s["case"]["page"]


def _weigh_plain(s):
    case = s["case"]
    y, token, real = _products(s)
    n = s["starts"][1:] - s["starts"][:-1]
    first = s["lengths"] - n
    i = torch.arange(s["max_new"], device="cuda", dtype=torch.int32)
    p = (first[:, None] + i)[:, :, None]
    j = torch.arange(y.shape[-1], device="cuda", dtype=torch.int32)
    seen = (j <= p) & real[:, :, None]
    if case["window"]:
        seen &= (j > p - case["window"]) | (j < case["sinks"])
    lse = s["lse"][token].view(case["seqs"], s["max_new"], case["kv_heads"], -1).permute(0, 2, 3, 1)
    y.sub_(lse.unsqueeze(-1)).exp_().masked_fill_(~seen[:, None, None], 0.0)
    got = y.sum((2, 3))                                                                # [sequences, kv heads, positions]
    seq, pos, at, row = _entries(s)
    old = s["weights"][at, :, row] * torch.where(pos < first[seq], case["decay"], 0.0)[:, None]
    s["weights"][at, :, row] = old + got[seq, :, pos]


def _evict_plain(s):
    case, page = s["case"], s["case"]["page"]
    B, H = case["seqs"], case["kv_heads"]
    seq, pos, at, row = _entries(s)
    rank = torch.full((B, s["max_length"], H), -math.inf, dtype=torch.float64, device="cuda")
    rank[seq, pos] = s["weights"][at, :, row].double().nan_to_num(-1e300, 1e300, -1e300)
    j = torch.arange(s["max_length"], device="cuda", dtype=torch.int32)
    length, keep = s["lengths"][:, None], s["keep"][:, None]
    sinks = torch.clamp(keep, max=case["sinks"])
    stays = (j < sinks) | ((j >= length - torch.clamp(keep - sinks, max=case["recent"])) & (j < length))
    rank.masked_fill_(stays[:, :, None], math.inf)
    order = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, : s["kept"].shape[2]]      # ties: the lowest position first
    k = torch.arange(s["kept"].shape[2], device="cuda", dtype=torch.int32)
    there = k < keep
    order = torch.sort(torch.where(there[:, :, None], order, s["max_length"]), dim=1).values
    s["kept"].copy_(torch.where(there[:, :, None], order, -1).transpose(1, 2))
    seq, k = torch.nonzero(there, as_tuple=True)
    src = order[seq, k]                                                                # [survivors, kv heads]
    at, row = s["table"][seq[:, None], src // page].long(), src % page
    to, to_row = s["to"][seq, k // page].long()[:, None], (k % page)[:, None]
    head = torch.arange(H, device="cuda")
    rows = [s[x][s["layer"]] for x in ("K_rows", "V_rows", "K_scales", "V_scales") if s[x] is not None] + [s["weights"]]
    [x.index_put_((to, head, to_row), x[at, head, row]) for x in rows]


# ---- the same from the definition, in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    new, lengths, page = _new(case), _lengths(case), case["page"]
    if case["kind"] in ("accept", "evict"):
        return None                                        # rows that move as they are
    if case["kind"] == "rotate":
        freq = [10000.0 ** (-i / case["pairs"]) for i in range(case["pairs"])]
        pos, out, i = _positions(case, seed).double(), {}, 0
        cos, sin = (torch.empty(sum(new), 1, case["pairs"], dtype=torch.float64, device="cuda") for _ in range(2))
        for axis, n in enumerate(_sections(case)):
            for i in range(i, i + n):
                cos[:, 0, i], sin[:, 0, i] = torch.cos(pos[axis] * freq[i]), torch.sin(pos[axis] * freq[i])
            i += 1
        first = [2 * i if case["adjacent"] else i for i in range(case["pairs"])]
        second = [2 * i + 1 if case["adjacent"] else i + case["pairs"] for i in range(case["pairs"])]

        def turned(x):
            y = x.double().clone()
            y[..., first] = x[..., first].double() * cos - x[..., second].double() * sin
            y[..., second] = x[..., first].double() * sin + x[..., second].double() * cos
            return y

        out = {"Q": turned(_queries(case, seed))}
        for k, name in enumerate(("K", "V")):
            x = _rows(case, seed, sum(new), k).to(_row_type(case))
            x = turned(x) if k == 0 else x.double()
            if case["store"] == "bf16":
                out[name + "_rows"] = None
            else:
                scale = (x.abs().amax(-1, keepdim=True) / 127.0).float().double()        # held in 32 bits
                out[name] = torch.where(scale > 0, torch.round(x / scale), torch.zeros_like(x)) * scale
                out[name + "_scales"] = None
        return out
    if work(case)["flops"] > 2.0e13:
        return None
    K = _logical(case, seed, 0)
    V = _logical(case, seed, 1) if case["kind"] == "tree" else None
    Q, group, H = _queries(case, seed), case["heads"] // case["kv_heads"], case["kv_heads"]
    number = lambda x, at, h: x[0][at, h].double() * (1.0 if x[1] is None else x[1][at, h].double()[:, None])  # noqa: E731
    if case["kind"] == "tree":
        O = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
        lse = torch.full(Q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
        for b, sees in enumerate(_ancestors(case, seed)):
            n, length, t0, r0 = new[b], lengths[b], sum(new[:b]), sum(lengths[:b])
            hidden = torch.zeros(n, length, dtype=torch.bool)
            hidden[:, length - n:] = True
            for i, js in enumerate(sees):
                hidden[i, [length - n + j for j in js]] = False
            hidden, at = hidden.cuda(), slice(r0, r0 + length)
            for h in range(H):
                k, v = number(K, at, h), number(V, at, h)
                for g in range(h * group, (h + 1) * group):
                    y = (Q[t0: t0 + n, g].double() @ k.T) / math.sqrt(case["d"])
                    y[hidden] = -math.inf
                    lse[t0: t0 + n, g] = torch.logsumexp(y, -1)
                    O[t0: t0 + n, g] = torch.exp(y - lse[t0: t0 + n, g, None]) @ v
        return {"O": O, "lse": lse}
    lse, old = _lse(case, seed).double(), _weights(case, seed, sum(lengths)).double()
    pages = sum(-(-l // page) for l in lengths) + 3
    order = torch.randperm(pages, generator=_generator(seed, 3), device="cuda")
    weights = torch.zeros(pages, H, page, dtype=torch.float64, device="cuda")
    at = 0
    for b, (n, length) in enumerate(zip(new, lengths)):
        t0, r0, first = sum(new[:b]), sum(lengths[:b]), length - n
        delta = (first + torch.arange(n, device="cuda"))[:, None] - torch.arange(length, device="cuda")[None]
        hidden = delta < 0
        if case["window"]:
            hidden |= (delta >= case["window"]) & (torch.arange(length, device="cuda")[None] >= case["sinks"])
        mine = old[r0: r0 + length] * case["decay"]
        mine[first:] = 0.0
        for g in range(case["heads"]):
            y = (Q[t0: t0 + n, g].double() @ number(K, slice(r0, r0 + length), g // group).T) / math.sqrt(case["d"])
            mine[:, g // group] += torch.exp(y - lse[t0: t0 + n, g, None]).masked_fill_(hidden, 0.0).sum(0)
        for p in range(0, length, page):
            weights[order[at], :, : min(page, length - p)] = mine[p: p + page].T
            at += 1
    return {"weights": weights}


def work(case):
    """Rows, queries, sums and outputs once each; of the cached rows those that some query sees; 4 d operations for each pair of a query
    and a key that it sees, 2 d where no values are summed.  Of a draft only the prefix and the tokens themselves are counted."""
    d, H, T = case["d"], case["kv_heads"], sum(_new(case))
    stored = d + 4 if case["store"] == "q8" else 2 * d
    size = 4 if case["rows"] == "f32" else 2
    if case["kind"] == "rotate":
        back = 2 * T * H * (stored + 2 * d) if case["store"] == "q8" else 0               # read back as bf16
        return {"bytes": T * case["heads"] * d * (size + 2) + 2 * T * H * (d * size + stored) + 4 * T * case["axes"] + back, "flops": 0}
    if case["kind"] == "tree":
        pairs = sum(n * (l - n) + n for n, l in zip(_new(case), _lengths(case)))
        return {"bytes": sum(_lengths(case)) * H * 2 * stored + T * case["heads"] * (4 * d + 4), "flops": 4 * d * case["heads"] * pairs}
    if case["kind"] == "accept":
        return {"bytes": sum(_accepted(case)) * case["layers"] * H * 4 * stored, "flops": 0}
    if case["kind"] == "weigh":
        pairs, rows = _visible(case)
        return {"bytes": H * (rows * stored + 8 * rows) + T * case["heads"] * (2 * d + 4), "flops": 2 * d * case["heads"] * pairs}
    kept = sum(_kept(case))
    return {"bytes": H * (4 * sum(_lengths(case)) + kept * (4 * stored + 8)), "flops": 0}
