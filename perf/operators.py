"""The operators of the paged cache of token sequences, as cases that can be timed and compared.

Beside the token maps of one image a model of this kind reads captions and writes text: sequences of any length, grouped key heads, a
prompt that arrives in chunks and tokens that arrive one by one.  Their keys and values lie in pages that a table assigns, as bf16 or
as 8-bit codes with one scale for each row.

  kind "write"   K and V rows of new tokens join the cache (quantised where it holds codes) and are read back as later steps see them
       "read"    cached rows of whole sequences are gathered (and turned into numbers again)
       "attend"  the new tokens' queries attend over the cache, which holds their keys too: O and the log-sum-exp of every row

A case names the cache (`store`, `d`, `kv_heads`, `page`), the batch (`seqs` sequences of up to `length` entries, `new` of them new;
`ragged`: lengths spread down to two fifths of that, new tokens likewise; `mixed`: two of three sequences bring a single token and one
brings none) and the mask (`causal`; `window` > 0: only the last `window` positions and the `sinks` first ones).  `rows` is the type
of the rows written or read.

The pool is laid out K rows, V rows, then for codes K scales, V scales, each [layer][page][kv head][row of the page].
"""
import math

import torch

own = False

LAYERS, LAYER = 2, 1       # the pool of a two-layer model; the second one is used
FIELDS = ("name", "kind", "store", "rows", "d", "heads", "kv_heads", "seqs", "new", "length", "ragged", "mixed", "causal", "window",
          "sinks", "page")


def _case(*values):
    return dict(zip(FIELDS, values))


def listed():
    return [
        # one new token for each of 8 sequences, grouped heads: what a generated token costs to store
        _case("write_tokens", "write", "q8", "bf16", 128, 32, 8, 8, 1, 1024, True, False, True, 0, 0, 64),
        # prompts of up to 4 096 tokens of a model with 16 heads
        _case("write_prompts", "write", "q8", "bf16", 128, 16, 16, 8, 4096, 4096, True, False, True, 0, 0, 128),
        # rows in single precision, small heads, small pages, odd lengths, a few tokens behind a longer past
        _case("write_odd", "write", "q8", "f32", 64, 12, 12, 7, 333, 1999, True, True, True, 0, 0, 16),
        # eight whole sequences as long as a 1024 x 1024 image's maps (10 521 tokens) brought back as bf16
        _case("read_whole", "read", "q8", "bf16", 128, 32, 8, 8, 10521, 10521, False, False, True, 0, 0, 64),
        # a few short ones in single precision
        _case("read_odd", "read", "q8", "f32", 64, 12, 4, 3, 211, 211, True, False, True, 0, 0, 16),
        # one user's next token behind a caption and a past answer: latency
        _case("token_one", "attend", "q8", "bf16", 128, 32, 8, 1, 1, 1999, False, False, True, 0, 0, 64),
        # the next token of 32 sequences of up to 10 521 entries: the serving step
        _case("token_batch", "attend", "q8", "bf16", 128, 32, 8, 32, 1, 10521, True, False, True, 0, 0, 64),
        # the next token behind a 4K-class image's 170 521 entries, 16 heads of their own, rows as they are
        _case("token_long", "attend", "bf16", "bf16", 128, 16, 16, 1, 1, 170521, False, False, True, 0, 0, 128),
        # 64 sequences that read 4 sinks and the last 1 024 positions only
        _case("token_window", "attend", "q8", "bf16", 128, 32, 8, 64, 1, 6000, True, False, True, 1024, 4, 32),
        # a 64 x 64 token map of two images over everything before it, every query sees all (no order inside a map)
        _case("map", "attend", "bf16", "bf16", 128, 16, 16, 2, 4096, 10521, False, False, False, 0, 0, 128),
        # a chunk of 2 048 prompt tokens of four sequences behind 6 144 cached ones
        _case("prompt", "attend", "q8", "bf16", 128, 32, 8, 4, 2048, 8192, False, False, True, 0, 0, 64),
        # continuous batching: chunks of odd lengths beside single tokens, window and sinks, small heads, small pages
        _case("mixed_window", "attend", "q8", "bf16", 64, 12, 4, 24, 777, 2999, True, True, True, 700, 5, 16),
    ]


def _spread(n, k):
    """n for k = 0, else between two fifths of it and all of it, evenly over k."""
    return max(1, round(n * (1.0 - 0.6 * ((k * 0.6180339887498949) % 1.0))))


def _new(case):
    if case["kind"] == "read":
        return _lengths(case)
    out = [_spread(case["new"], b) if case["ragged"] else case["new"] for b in range(case["seqs"])]
    if case["mixed"]:
        out = [0 if b == 4 else (n if b % 3 == 0 else 1) for b, n in enumerate(out)]
    return out


def _lengths(case):
    out = [_spread(case["length"], b) if case["ragged"] else case["length"] for b in range(case["seqs"])]
    return out if case["kind"] == "read" else [max(l, n) for l, n in zip(out, _new(case))]


def _visible(case):
    """(query, key) pairs that a head's mask leaves, and cached rows that some query sees."""
    pairs = rows = 0
    for n, length in zip(_new(case), _lengths(case)):
        if not n:
            continue
        first = length - n
        w, sinks = case["window"], case["sinks"]
        lo = max(0, first - w + 1) if w and case["causal"] else (max(0, first - w + 1) if w else 0)
        rows += length - lo + min(sinks if w else 0, lo)
        for i in range(n):
            p = first + i
            hi = p + 1 if case["causal"] else length
            start = max(0, p - w + 1) if w else 0
            pairs += hi - start + min(sinks if w else 0, start)
    return pairs, rows


def draw(rng):
    """One more case: any cache, batch and mask, from one token to chunks of thousands, odd sizes among them."""
    def log(lo, hi):
        return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))

    while True:
        kind = rng.choice(["write", "read", "attend", "attend", "attend"])
        store, d = rng.choice(["q8", "q8", "bf16"]), rng.choice([64, 128, 128])
        kv_heads, group = rng.choice([1, 2, 4, 5, 8, 16]), rng.choice([1, 1, 2, 3, 4, 8])
        length = log(1, 40000)
        new = 1 if kind == "attend" and rng.random() < 0.4 else log(1, min(length, 4096))
        window = log(16, 4096) if kind == "attend" and rng.random() < 0.3 else 0
        case = {"kind": kind, "store": store, "rows": "bf16" if kind == "attend" else rng.choice(["bf16", "bf16", "f32"]), "d": d,
                "heads": kv_heads * group, "kv_heads": kv_heads, "seqs": log(1, 64), "new": length if kind == "read" else new,
                "length": length, "ragged": rng.random() < 0.7, "mixed": kind != "read" and new > 1 and rng.random() < 0.3,
                "causal": kind != "attend" or rng.random() < 0.75, "window": window, "sinks": rng.choice([0, 1, 4, 16]) if window else 0,
                "page": rng.choice([16, 32, 64, 64, 128])}
        w = work(case)
        scores = case["seqs"] * case["heads"] * max(_new(case)) * max(_lengths(case)) if kind == "attend" else 0
        held = 8 * case["seqs"] * max(_lengths(case)) * kv_heads * d
        if w["flops"] <= 8.0e11 and w["bytes"] <= 1.3e9 and scores <= 2.0e9 and held <= 8.0e9 and sum(_new(case)) > 0:
            return case


# ---- inputs -----------------------------------------------------------------------------------------------------------------------
def _generator(seed, k):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 0x9E3779B1 + k * 0x85EBCA6B + 12345) & 0x7FFFFFFFFFFFFFFF)
    return g


def _rows(case, seed, n, what):
    """[n, kv heads, d] K or V rows: the keys of a head share an offset, every 512th one is a sink with four times the length."""
    g = _generator(seed, what)
    x = torch.randn(n, case["kv_heads"], case["d"], generator=g, device="cuda")
    if what == 0:
        x += 0.5 * torch.randn(1, case["kv_heads"], case["d"], generator=g, device="cuda")
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
    g = _generator(seed, 2)
    return torch.randn(sum(_new(case)), case["heads"], case["d"], generator=g, device="cuda").bfloat16()


def _starts(counts):
    return torch.tensor([sum(counts[:b]) for b in range(len(counts) + 1)], dtype=torch.int32, device="cuda")


def _region_bytes(case, pages):
    """Bytes of the K rows (or V rows) and of the K scales (or V scales)."""
    rows = LAYERS * pages * case["kv_heads"] * case["page"]
    return rows * case["d"] * (1 if case["store"] == "q8" else 2), rows * 4 if case["store"] == "q8" else 0


def prepare(case, seed):
    new, lengths, page = _new(case), _lengths(case), case["page"]
    need = [-(-l // page) for l in lengths]
    pages, g = sum(need) + 3, _generator(seed, 3)
    order = torch.randperm(pages, generator=g, device="cuda")[: sum(need)].to(torch.int32)      # pages were handed out in no order
    table = torch.full((case["seqs"], max(need)), -1, dtype=torch.int32, device="cuda")
    for b, n in enumerate(need):
        table[b, :n] = order[sum(need[:b]): sum(need[: b + 1])]
    rows_bytes, scale_bytes = _region_bytes(case, pages)
    pool = torch.zeros(2 * rows_bytes + 2 * scale_bytes, dtype=torch.uint8, device="cuda")
    shape = (LAYERS, pages, case["kv_heads"], page)
    dt = torch.int8 if case["store"] == "q8" else torch.bfloat16
    s = {"case": case, "pool": pool, "table": table, "lengths": torch.tensor(lengths, dtype=torch.int32, device="cuda"),
         "starts": _starts(new), "max_new": max(new), "max_length": max(lengths), "tokens": sum(new)}
    for i, name in enumerate(("K", "V")):
        s[name + "_rows"] = pool[i * rows_bytes: (i + 1) * rows_bytes].view(dt).view(*shape, case["d"])
        at = 2 * rows_bytes + i * scale_bytes
        s[name + "_scales"] = pool[at: at + scale_bytes].view(torch.float32).view(shape) if scale_bytes else None
    if case["kind"] == "write":
        s["K"], s["V"] = (_rows(case, seed, sum(new), i).to(_row_type(case)) for i in (0, 1))
    else:
        pos = torch.cat([torch.arange(l, device="cuda") for l in lengths])
        seq = torch.repeat_interleave(torch.arange(case["seqs"], device="cuda"), s["lengths"].long())
        at, row = table[seq, pos // page].long(), pos % page
        for i, name in enumerate(("K", "V")):
            codes, scales = _logical(case, seed, i)
            s[name + "_rows"][LAYER, at, :, row] = codes
            if scales is not None:
                s[name + "_scales"][LAYER, at, :, row] = scales
    shape = (sum(new), case["kv_heads"], case["d"])
    if case["kind"] == "attend":
        s["Q"] = _queries(case, seed)
        s["O"], s["lse"] = torch.empty_like(s["Q"]), torch.empty(s["Q"].shape[:2], device="cuda")
    else:
        s["K_out"], s["V_out"] = (torch.empty(shape, dtype=_row_type(case), device="cuda") for _ in range(2))
    if own:
        from paper_2505_19602_b200 import binding

        s["kv"] = binding.PagedKV(LAYERS, pages, case["kv_heads"], case["d"], store=case["store"], page_tokens=page, pool=pool)
        s["batch"] = binding.PagedBatch(table, s["lengths"], s["starts"], s["tokens"], s["max_new"], s["max_length"])
    return s


# ---- one pass ---------------------------------------------------------------------------------------------------------------------
def run(s):
    case = s["case"]
    if case["kind"] == "write":
        if own:
            s["kv"].scalekv_paged_write(LAYER, s["batch"], s["K"], s["V"])
            s["kv"].scalekv_paged_read(LAYER, s["batch"], s["K_out"], s["V_out"])
            K, V = s["K_out"], s["V_out"]
        else:
            _write_plain(s, "K")
            _write_plain(s, "V")
            K, V = _read_plain(s, "K"), _read_plain(s, "V")
        if case["store"] == "bf16":
            return {"K": K, "V": V, "K_rows": s["K_rows"], "V_rows": s["V_rows"]}
        return {"K": K, "V": V, "K_scales": s["K_scales"], "V_scales": s["V_scales"]}
    if case["kind"] == "read":
        if own:
            s["kv"].scalekv_paged_read(LAYER, s["batch"], s["K_out"], s["V_out"])
            return {"K": s["K_out"], "V": s["V_out"]}
        return {"K": _read_plain(s, "K"), "V": _read_plain(s, "V")}
    if own:
        s["kv"].scalekv_paged_attend(LAYER, s["batch"], s["Q"], s["O"], lse=s["lse"], causal=case["causal"], window=case["window"],
                                     n_sink=case["sinks"])
        return {"O": s["O"], "lse": s["lse"]}
    O, lse = _attend_plain(s)
    return {"O": O, "lse": lse}


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


def _write_plain(s, name):
    x, (at, row) = s[name].float(), _where(s)
    if s["case"]["store"] == "bf16":
        s[name + "_rows"][LAYER, at, :, row] = x.bfloat16()
        return
    a = x.abs().amax(-1)
    scale = a / torch.full_like(a, 127.0)
    codes = torch.where(scale.unsqueeze(-1) > 0, x / scale.unsqueeze(-1), torch.zeros_like(x)).round().clamp(-127, 127)
    s[name + "_rows"][LAYER, at, :, row] = codes.to(torch.int8)
    s[name + "_scales"][LAYER, at, :, row] = scale


def _read_plain(s, name):
    at, row = _where(s)
    x = s[name + "_rows"][LAYER, at, :, row].float()
    if s["case"]["store"] == "q8":
        x = x * s[name + "_scales"][LAYER, at, :, row].unsqueeze(-1)
    return x.to(_row_type(s["case"]))


def _gather_plain(s, name):
    """[sequences, kv heads, positions, d] in 32 bits, the table's holes from page 0 (no query sees them)."""
    table = s["table"].clamp(min=0).long()
    x = s[name + "_rows"][LAYER][table].float()
    if s["case"]["store"] == "q8":
        x = x * s[name + "_scales"][LAYER][table].unsqueeze(-1)
    return x.transpose(1, 2).flatten(2, 3)


def _attend_plain(s):
    case = s["case"]
    B, H, G, N = case["seqs"], case["kv_heads"], case["heads"] // case["kv_heads"], s["max_new"]
    n = s["starts"][1:] - s["starts"][:-1]
    i = torch.arange(N, device="cuda", dtype=torch.int32)
    from_token = (s["starts"][:-1, None] + i).clamp(max=s["tokens"] - 1).long()
    Q = s["Q"][from_token].float().view(B, N, H, G, case["d"]).permute(0, 2, 3, 1, 4).reshape(B, H, G * N, case["d"])
    K = _gather_plain(s, "K")
    y = torch.matmul(Q, K.transpose(2, 3)).view(B, H, G, N, -1).mul_(1.0 / math.sqrt(case["d"]))
    p = (s["lengths"][:, None] - n[:, None] + i)[:, :, None]                          # a query's position
    j = torch.arange(y.shape[-1], device="cuda", dtype=torch.int32)
    seen = j < s["lengths"][:, None, None]
    if case["causal"]:
        seen = seen & (j <= p)
    if case["window"]:
        seen = seen & ((j > p - case["window"]) | (j < case["sinks"]))
    y.masked_fill_(~seen[:, None, None], -math.inf)
    top = y.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    y.sub_(top).exp_()
    total = y.sum(-1, keepdim=True)
    lse = (top + total.log()).view(B, H, G, N)
    O = torch.matmul(y.view(B, H, G * N, -1), _gather_plain(s, "V")).view(B, H, G, N, -1)
    O = torch.where(total > 0, O / total, torch.zeros_like(O))
    seq, place = _tokens(s)
    O = O.permute(0, 3, 1, 2, 4).reshape(B, N, H * G, case["d"])[seq, place.long()]
    return O.bfloat16(), lse.permute(0, 3, 1, 2).reshape(B, N, H * G)[seq, place.long()].contiguous()


# ---- the same from the definition, in 64 bits --------------------------------------------------------------------------------------
def exact(case, seed):
    new, lengths = _new(case), _lengths(case)
    if case["kind"] == "write":
        out = {}
        for k, name in enumerate(("K", "V")):
            x = _rows(case, seed, sum(new), k).to(_row_type(case)).double()
            if case["store"] == "bf16":
                out[name] = x.float().bfloat16().double()
            else:
                scale = (x.abs().amax(-1, keepdim=True) / 127.0).float().double()        # held in 32 bits
                out[name] = torch.where(scale > 0, torch.round(x / scale), torch.zeros_like(x)) * scale
            out[name + ("_rows" if case["store"] == "bf16" else "_scales")] = None
        return out
    stored = [_logical(case, seed, k) for k in (0, 1)]
    if case["kind"] == "read":
        return {name: x.double() if scales is None else x.double() * scales.double().unsqueeze(-1)
                for name, (x, scales) in zip(("K", "V"), stored)}
    if work(case)["flops"] > 2.0e13:
        return None
    Q, group = _queries(case, seed), case["heads"] // case["kv_heads"]
    O = torch.zeros(Q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(Q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, (n, length) in enumerate(zip(new, lengths)):
        t0, r0 = sum(new[:b]), sum(lengths[:b])
        if n == 0:
            continue
        for h in range(case["kv_heads"]):
            k, v = (x[r0: r0 + length, h].double() * (1.0 if scales is None else scales[r0: r0 + length, h].double()[:, None])
                    for x, scales in stored)
            for g in range(h * group, (h + 1) * group):
                y = (Q[t0: t0 + n, g].double() @ k.T) / math.sqrt(case["d"])
                delta = (length - n + torch.arange(n, device="cuda"))[:, None] - torch.arange(length, device="cuda")[None]
                hidden = torch.zeros_like(delta, dtype=torch.bool)
                if case["causal"]:
                    hidden |= delta < 0
                if case["window"]:
                    hidden |= (delta >= case["window"]) & (torch.arange(length, device="cuda")[None] >= case["sinks"])
                y[hidden] = -math.inf
                lse[t0: t0 + n, g] = torch.logsumexp(y, -1)
                O[t0: t0 + n, g] = torch.nan_to_num(torch.exp(y - lse[t0: t0 + n, g, None])) @ v
    return {"O": O, "lse": lse}


def work(case):
    """Rows, queries and outputs once each; of the cached rows those that some query sees; 4 d operations for each pair of a query
    and a key that it sees."""
    d, H, T = case["d"], case["kv_heads"], sum(_new(case))
    stored = d + 4 if case["store"] == "q8" else 2 * d
    size = 4 if case["rows"] == "f32" else 2
    if case["kind"] == "attend":
        pairs, rows = _visible(case)
        return {"bytes": rows * H * 2 * stored + T * case["heads"] * (4 * d + 4), "flops": 4 * d * case["heads"] * pairs}
    given = 2 * T * H * d * size                       # rows in, or out
    if case["kind"] == "write":
        return {"bytes": 2 * given + 2 * T * H * stored, "flops": 0}
    return {"bytes": given + 2 * T * H * stored, "flops": 0}
