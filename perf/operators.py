"""Operators of a paged K/V cache: the measured cases, their plain forms and the calls that a server makes of them.

  rows     cascade_rope_rows                           rows of a ragged batch turned by their own positions
  table    cascade_rope_table_scaled                   the positional table of a model whose angles were stretched for long contexts
  append   cascade_paged_append                        new rows go to the pages of their sequences, turned on the way, with their queries
  attn     cascade_attn_paged                          attention of the new rows over the pages: chunks, single tokens, other lengths
  fork     cascade_pages_fork, cascade_pages_copy      a step of the page tables: sequences forked, ended and given room
  compact  cascade_pages_compact, cascade_pages_copy   live pages moved together at the front of the pool

Shapes as in the library: pages [n_pages, page_size, kv_heads, head_dim], rows [rows, heads, head_dim], page tables int32
[sequences, pages], row_start int32 [sequences + 1], kv_len int32 [sequences] (rows of the cache, the new ones counted).
"""
import math

import numpy as np
import torch

own = False


def _case(name, op, **more):
    c = dict(op=op, **more)
    return dict(c, name=name) if name else c


def _attn(name, B, rows, kv, H, Hkv, d, page, dtype="bf16", causal=True):
    return _case(name, "attn", B=B, rows_lo=rows[0], rows_hi=rows[1], kv_lo=kv[0], kv_hi=kv[1], H=H, Hkv=Hkv, d=d, page=page,
                 dtype=dtype, causal=causal)


def _append(name, B, rows, kv, H, Hkv, d, page, rot, interleaved, dtype="bf16"):
    return _case(name, "append", B=B, rows_lo=rows[0], rows_hi=rows[1], kv_lo=kv[0], kv_hi=kv[1], H=H, Hkv=Hkv, d=d, page=page,
                 rot=rot, interleaved=interleaved, dtype=dtype)


def _rows(name, n, H, d, rot, interleaved, far, dtype, padded):
    return _case(name, "rows", n=n, H=H, d=d, rot=rot, interleaved=interleaved, far=far, dtype=dtype, padded=padded)


def _table(name, n, rot, kind, factor):
    return _case(name, "table", n=n, rot=rot, kind=kind, factor=factor)


def _fork(name, groups, beams, kv, page, layers, Hkv, d, spare):
    return _case(name, "fork", groups=groups, beams=beams, kv_lo=kv[0], kv_hi=kv[1], page=page, layers=layers, Hkv=Hkv, d=d,
                 spare=spare, add=1)


def _compact(name, groups, beams, kv, page, layers, Hkv, d, spare):
    return _case(name, "compact", groups=groups, beams=beams, kv_lo=kv[0], kv_hi=kv[1], page=page, layers=layers, Hkv=Hkv, d=d,
                 spare=spare)


def listed():
    return [
        # The table of a model whose context was stretched sixteen times: built when the server starts.
        _table("table_32k_ramp", 32768, 128, "ramp", 16.0),
        # Query rows of a mixed batch, neighbouring columns paired, half the head turned, positions far into the context.
        _rows("rows_4099_interleaved_part", 4099, 32, 128, 64, True, 32768, "bf16", False),
        # One generated token for each of 64 requests: rotate q and k, append k and v.  Latency.
        _append("append_decode_b64", 64, (1, 1), (100, 16384), 32, 8, 128, 64, 128, False),
        # Chunks of four prompts on their way into the cache.
        _append("append_chunk_4_ragged", 4, (300, 1021), (1200, 8192), 32, 8, 128, 16, 64, True),
        # One user's token in the middle of a long chat: the smallest call there is.
        _attn("decode_2500_b1", 1, (1, 1), (2500, 2500), 32, 8, 128, 64),
        # A full decode batch, requests of very different lengths: bound by the reads of the cache.
        _attn("decode_16k_b64_ragged", 64, (1, 1), (1000, 16384), 32, 8, 128, 64),
        # One chunk of a chunked prefill near the end of 7168 rows.
        _attn("chunk_512_of_7k", 1, (512, 512), (7168, 7168), 32, 8, 128, 64),
        # A step that mixes single tokens, drafts and chunks, heads of 64 columns, small pages.
        _attn("mixed_16_d64", 16, (1, 701), (40, 3001), 16, 4, 64, 16),
        # A decoder's rows over the encoder's states of another length, fp32, bidirectional.
        _attn("cross_8_f32", 8, (17, 128), (60, 512), 12, 12, 64, 16, "f32", False),
        # The largest: a long chunk of a document of 16384 tokens.
        _attn("chunk_2048_of_16k", 1, (2048, 2048), (16384, 16384), 32, 8, 128, 128),
        # A beam step of 16 requests with four beams each: beams forked, ended, one token of room for each.
        _fork("fork_16x4", 16, 4, (33, 900), 16, 8, 8, 128, 200),
        # A pool with holes is closed up before it shrinks.
        _compact("compact_2500_pages", 32, 4, (200, 900), 16, 8, 8, 128, 1600),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["rows", "table", "append", "attn", "attn", "attn", "attn", "fork", "compact"])
    page = rng.choice([16, 32, 48, 64, 128])
    if op == "table":
        rot = rng.choice([16, 32, 64, 96, 128])
        return _table(None, _log_int(rng, 64, 32768), rot, rng.choice(["none", "linear", "base", "bands", "ramp"]), rng.choice([2.0, 4.0, 8.0, 32.0]))
    if op == "rows":
        d = rng.choice([64, 128])
        return _rows(None, _log_int(rng, 1, 4096), rng.choice([1, 4, 8, 12, 32]), d, rng.choice([16, d // 2, d]), rng.random() < 0.5,
                     _log_int(rng, 64, 32768), rng.choice(["bf16", "bf16", "f32"]), rng.random() < 0.3)
    if op in ("fork", "compact"):
        groups, beams = _log_int(rng, 1, 32), rng.choice([1, 2, 4])
        lo = _log_int(rng, 10, 400)
        make = _fork if op == "fork" else _compact
        return make(None, groups, beams, (lo, lo + _log_int(rng, 1, 500)), rng.choice([16, 32]), rng.choice([1, 2, 4]), rng.choice([4, 8]),
                    rng.choice([64, 128]), _log_int(rng, 160, 1000))
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    d = rng.choice([128, 128, 64])
    H, Hkv = rng.choice([(32, 8), (16, 4), (12, 12), (16, 8), (8, 1), (64, 8)])
    form = rng.choice(["decode", "draft", "chunk", "mixed"])
    hi = _log_int(rng, 64, 12000)
    lo = rng.randrange(max(1, hi // 8), hi + 1)
    if form == "decode":
        B, rows = _log_int(rng, 1, max(1, min(64, 300000 // hi))), (1, 1)
    elif form == "draft":
        B, rows = _log_int(rng, 1, max(1, min(32, 100000 // hi))), (2, 6)
    elif form == "chunk":
        B, n = rng.choice([1, 1, 2, 3]), _log_int(rng, 16, 700)
        rows = (n, n)
    else:
        B, rows = _log_int(rng, 2, 8), (1, _log_int(rng, 8, 400))
    if op == "append":
        return _append(None, B, rows, (lo, hi), H, Hkv, d, page, rng.choice([32, d // 2, d]), rng.random() < 0.5, dtype)
    if dtype == "f32" or B > 4:
        lo, hi = min(lo, 4000), min(hi, 4000)
    return _attn(None, B, rows, (lo, hi), H, Hkv, d, page, dtype, rng.random() < 0.75)


# ---------------------------------------------------------------------------------------------------- sizes that follow from a case

def _spread(lo, hi, n):
    """n whole numbers between lo and hi, the last of them hi."""
    return [int(round(lo + (hi - lo) * ((1 + (n - 1 - i) * 0.6180339887) % 1.0 if i < n - 1 else 1.0))) for i in range(n)]


def _lengths(case):
    rows = _spread(case["rows_lo"], case["rows_hi"], case["B"])
    kv = [max(1, k) for k in _spread(case["kv_lo"], case["kv_hi"], case["B"])]
    if case["op"] == "append" or case["causal"]:
        kv = [max(k, n) for k, n in zip(kv, rows)]
    return rows, kv


def _beams(case):
    """(rows, pages of the group's common prefix, pages) of every group's beams; which beam each new one continues."""
    kv = _spread(case["kv_lo"], case["kv_hi"], case["groups"])
    shared = [k // 2 // case["page"] for k in kv]
    pages = [-(-k // case["page"]) for k in kv]
    n = case["beams"]
    source = [-1 if g % 7 == 6 else g * n + j // 2 for g in range(case["groups"]) for j in range(n)]
    return kv, shared, pages, source


def _pages_in_use(case):
    _, shared, pages, _ = _beams(case)
    return sum(s + case["beams"] * (p - s) for s, p in zip(shared, pages))


def work(case):
    op, es = case["op"], 4 if case.get("dtype") == "f32" else 2
    if op == "table":
        return {"bytes": case["n"] * case["rot"] * 4, "flops": case["n"] * case["rot"] // 2 * 40}
    if op == "rows":
        rows = case["n"] * case["H"]
        return {"bytes": 2 * rows * case["d"] * es + case["n"] * (case["rot"] * 4 + 4), "flops": rows * case["rot"] * 3}
    if op in ("fork", "compact"):
        used = _pages_in_use(case)
        n_pages, n = used + case["spare"], case["groups"] * case["beams"]
        kv, _, pages, source = _beams(case)
        if op == "fork":  # a copy for every second beam that ends inside a page
            copies = sum(1 for i, s in enumerate(source) if s >= 0 and i % case["beams"] % 2 == 1 and kv[i // case["beams"]] % case["page"])
            used = sum(1 for s in source if s >= 0) * max(pages)
        else:
            copies = used * case["spare"] // n_pages
        table = n * (max(pages) + 1)
        page = case["page"] * case["Hkv"] * case["d"] * 2
        return {"bytes": 4 * (2 * table + n_pages) + 2 * copies * page * 2 * case["layers"], "flops": n_pages + 2 * table}
    rows, kv = _lengths(case)
    H, Hkv, d = case["H"], case["Hkv"], case["d"]
    if op == "append":
        n = sum(rows)
        return {"bytes": n * (2 * (H + 2 * Hkv) * d * es + case["rot"] * 4) + 4 * len(rows) * 3, "flops": n * (H + Hkv) * case["rot"] * 3}
    n, P = sum(rows), case["page"]
    pairs = sum(r * k - (r * (r - 1) // 2 if case["causal"] else 0) for r, k in zip(rows, kv))
    nbytes = n * H * (2 * d * es + 4) + sum(2 * k * Hkv * d * es + 4 * -(-k // P) for k in kv)
    return {"bytes": nbytes, "flops": 4 * d * H * pairs}


# ---------------------------------------------------------------------------------------------------- inputs

def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(int(seed))


def _int(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _place(counts, n_pages, width, rng):
    """A page table in which sequence i has counts[i] pages, taken from anywhere in the pool."""
    ids = rng.permutation(n_pages)
    table, at = np.full((len(counts), width), -1, np.int32), 0
    for i, c in enumerate(counts):
        table[i, :c] = ids[at:at + c]
        at += c
    return table


def _prepare_beams(case, seed, gen):
    rng = np.random.default_rng([seed, 11])
    kv, shared, pages, source = _beams(case)
    n_pages, beams, width = _pages_in_use(case) + case["spare"], case["beams"], max(pages) + 1
    ids, at = rng.permutation(n_pages), 0
    table = np.full((case["groups"] * beams, width), -1, np.int32)
    for g in range(case["groups"]):
        s, p = shared[g], pages[g]
        table[g * beams:(g + 1) * beams, :s] = ids[at:at + s]
        at += s
        for j in range(beams):
            table[g * beams + j, s:p] = ids[at:at + p - s]
            at += p - s
    pool = torch.empty((case["layers"], 2, n_pages, case["page"], case["Hkv"], case["d"]), dtype=torch.bfloat16, device="cuda")
    pool.normal_(generator=gen)
    return dict(case=case, n_pages=n_pages, table=_int(table), kv_len=_int([k for k in kv for _ in range(beams)]), pool=pool,
                pools=[pool[layer, j] for layer in range(case["layers"]) for j in range(2)], source=_int(source),
                add=_int([case.get("add", 0) if s >= 0 else 0 for s in source]))


def _angles(n, rot, base, kind, factor, original, low, high):
    """The angles of every position, in 64 bits, and the factor on cosine and sine."""
    i = torch.arange(0, rot, 2, dtype=torch.float64, device="cuda")
    theta, scale = base ** (-i / rot), 1.0
    if kind == "linear":
        theta = theta / factor
    elif kind == "base":
        theta = (base * factor ** (rot / (rot - 2))) ** (-i / rot)
    elif kind == "bands":
        turns = original * theta / (2 * math.pi)
        keep = ((turns - low) / (high - low)).clamp(0, 1)
        theta = theta * keep + theta / factor * (1 - keep)
    elif kind == "ramp":
        where = lambda r: rot * math.log(original / (2 * math.pi * r)) / (2 * math.log(base))  # noqa: E731
        a, b = max(math.floor(where(high)), 0), min(math.ceil(where(low)), rot - 1)
        far = ((torch.arange(rot // 2, dtype=torch.float64, device="cuda") - a) / max(b - a, 0.001)).clamp(0, 1)
        theta, scale = theta * (1 - far) + theta / factor * far, 0.1 * math.log(factor) + 1
    return torch.arange(n, dtype=torch.float64, device="cuda")[:, None] * theta, scale


def prepare(case, seed):
    gen, rng, op = _gen(seed), np.random.default_rng([seed, 7]), case["op"]
    if op == "table":
        return dict(case=case, base=10000.0 * (1 + seed % 64), original=4096.0, low=1.0, high=32.0 if case["kind"] == "ramp" else 4.0)
    if op in ("fork", "compact"):
        return _prepare_beams(case, seed, gen)
    dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)

    def turns(n, rot):  # the program's positional table
        angle, _ = _angles(n, rot, 500000.0, "none", 1.0, 0, 0, 0)
        return torch.stack([angle.cos(), angle.sin()], -1).float()

    if op == "rows":
        positions = rng.integers(0, case["far"], case["n"])
        if case["padded"]:
            positions[case["n"] - case["n"] // 4:] = -1
        x = normal(case["n"], case["H"], case["d"])
        return dict(case=case, x=x, positions=_int(positions), turns=turns(case["far"], case["rot"]), y=torch.zeros_like(x))
    rows, kv = _lengths(case)
    P, H, Hkv, d, n = case["page"], case["H"], case["Hkv"], case["d"], sum(rows)
    counts = [-(-k // P) for k in kv]
    n_pages = sum(counts) + 8
    pages = torch.empty((2, n_pages, P, Hkv, d), dtype=dtype, device="cuda")
    pages.normal_(generator=gen)
    s = dict(case=case, q=normal(n, H, d), k_pages=pages[0], v_pages=pages[1], max_rows=max(rows), max_kv=max(kv), scale=1 / math.sqrt(d),
             table=_int(_place(counts, n_pages, max(counts), rng)), row_start=_int(np.concatenate([[0], np.cumsum(rows)])), kv_len=_int(kv))
    s["out"] = torch.empty_like(s["q"])
    if op == "append":
        s.update(k=normal(n, Hkv, d), v=normal(n, Hkv, d), turns=turns(max(kv), case["rot"]))
    return s


# ---------------------------------------------------------------------------------------------------- one pass

def run(s):
    case, op = s["case"], s["case"]["op"]
    if own:
        from paper_2507_05228_b200 import binding as cb
        if op == "table":
            return cb.cascade_rope_table_scaled(case["n"], case["rot"], s["base"], case["kind"], case["factor"], s["original"], s["low"], s["high"])
        if op == "rows":
            return cb.cascade_rope_rows(s["x"], s["positions"], s["turns"], interleaved=case["interleaved"], out=s["y"])
        if op == "append":
            q = cb.cascade_paged_append(s["k"], s["v"], s["k_pages"], s["v_pages"], s["table"], s["row_start"], s["kv_len"], q=s["q"],
                                        rope_table=s["turns"], interleaved=case["interleaved"], q_out=s["out"])
            return q, s["k_pages"], s["v_pages"]
        if op == "attn":
            return cb.cascade_attn_paged(s["q"], s["k_pages"], s["v_pages"], s["table"], s["row_start"], s["kv_len"], s["scale"],
                                         causal=case["causal"], max_rows=s["max_rows"], out=s["out"])
        if op == "fork":
            table, kv_len, refs, copies, report = cb.cascade_pages_fork(s["table"], s["kv_len"], s["source"], s["add"], s["n_pages"], case["page"])
            cb.cascade_pages_copy(s["pools"], copies)
            return table, kv_len, refs, copies, report, s["pool"]
        table, refs, moves, report = cb.cascade_pages_compact(s["table"], s["kv_len"], s["n_pages"], case["page"])
        cb.cascade_pages_copy(s["pools"], moves)
        return table, refs, moves, report, s["pool"]
    if op == "table":
        angle, scale = _angles(case["n"], case["rot"], s["base"], case["kind"], case["factor"], s["original"], s["low"], s["high"])
        return (torch.stack([angle.cos(), angle.sin()], -1) * scale).float()
    if op == "rows":
        there = s["positions"] >= 0
        turned = _turn(s["x"].float(), s["turns"][s["positions"].clamp(min=0)], case["rot"], case["interleaved"])
        return torch.where(there[:, None, None], turned.to(s["x"].dtype), s["y"])
    return {"append": _plain_append, "attn": _plain_attn, "fork": _plain_fork, "compact": _plain_compact}[op](s)


def _turn(x, cs, rot, interleaved):
    """x [rows, heads, d] with its first `rot` columns turned by cs [rows, rot / 2, 2]."""
    cos, sin = cs[:, None, :, 0], cs[:, None, :, 1]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if interleaved else (x[..., :rot // 2], x[..., rot // 2:rot])
    lo, hi = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([lo, hi], -1).flatten(-2) if interleaved else torch.cat([lo, hi], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(s):
    case, first, kv_len = s["case"], s["row_start"].long(), s["kv_len"].long()
    row = torch.arange(s["q"].shape[0], device="cuda")
    b = (row[:, None] >= first[None, 1:]).sum(1)  # whose row it is
    y = kv_len[b] - first[b + 1] + row
    page, slot, cs = s["table"].long()[b, y // case["page"]], y % case["page"], s["turns"][y]
    s["k_pages"][page, slot] = _turn(s["k"].float(), cs, case["rot"], case["interleaved"]).to(s["k"].dtype)
    s["v_pages"][page, slot] = s["v"]
    q = _turn(s["q"].float(), cs, case["rot"], case["interleaved"]).to(s["q"].dtype)
    return q, s["k_pages"], s["v_pages"]


def _plain_attn(s):
    case, q, first, kv_len = s["case"], s["q"], s["row_start"].long(), s["kv_len"].long()
    H, Hkv, d, P, B, most = case["H"], case["Hkv"], case["d"], case["page"], case["B"], s["max_rows"]
    n_kv, G, n = s["table"].shape[1] * P, H // Hkv, q.shape[0]
    of = first[:-1, None] + torch.arange(most, device="cuda")  # the rows of each sequence side by side
    there = of < first[1:, None]
    y = torch.arange(n_kv, device="cuda")
    sees = kv_len[:, None].expand(B, most)
    if case["causal"]:
        sees = kv_len[:, None] - first[1:, None] + of + 1
    in_cache = (y < kv_len[:, None])[:, :, None, None]
    table = s["table"].long().clamp(min=0)
    k = s["k_pages"][table].reshape(B, n_kv, Hkv, d).float()
    v = s["v_pages"][table].reshape(B, n_kv, Hkv, d).float()
    k, v = torch.where(in_cache, k, 0), torch.where(in_cache, v, 0)
    rows = q.float()[of.clamp(max=n - 1)].reshape(B, most, Hkv, G, d).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * most, d)
    logits = (rows @ k.permute(0, 2, 3, 1)).view(B, Hkv, G, most, n_kv) * s["scale"]
    logits = logits.masked_fill((y >= sees[:, :, None])[:, None, None], -math.inf)
    m = logits.amax(-1, keepdim=True)
    m = torch.where(m == -math.inf, 0, m)
    logits = (logits - m).exp()
    total = logits.sum(-1, keepdim=True)
    o = (logits.view(B, Hkv, G * most, n_kv) @ v.transpose(1, 2)).view(B, Hkv, G, most, d) / torch.where(total > 0, total, 1)
    lse = (m + total.log())[..., 0]
    to = torch.where(there, of, n)  # rows past a sequence's end go to a row that is dropped
    out, stat = o.new_empty(n + 1, H, d), lse.new_empty(n + 1, H)
    out[to] = o.permute(0, 3, 1, 2, 4).reshape(B, most, H, d)
    stat[to] = lse.permute(0, 3, 1, 2).reshape(B, most, H)
    return out[:n].to(q.dtype), stat[:n]


def _copy_pages(pool, pairs):
    """Pages pairs[:, 0] of every layer to pages pairs[:, 1]; -1: none."""
    there = (pairs[:, 0] >= 0).nonzero()[:, 0]
    pool[:, :, pairs[there, 1].long()] = pool[:, :, pairs[there, 0].long()]


def _plain_fork(s):
    case, n_pages, P, dev = s["case"], s["n_pages"], s["case"]["page"], "cuda"
    source, add = s["source"].long(), s["add"].long()
    n, width = s["table"].shape
    live, me, col = source >= 0, torch.arange(n, device=dev), torch.arange(width, device=dev)
    had = torch.where(live, s["kv_len"].long()[source.clamp(min=0)], 0)
    old, new = -(-had // P), -(-(had + add) // P)
    pages = s["table"].long()[source.clamp(min=0)]
    kept = col < old[:, None]
    dump = torch.where(kept, pages, n_pages)  # a last place for what is none
    holders = torch.zeros(n_pages + 1, dtype=torch.long, device=dev).scatter_add_(0, dump.flatten(), kept.long().flatten())
    writes = live & (add > 0) & (had % P > 0)
    last = torch.where(writes, pages.gather(1, (old - 1).clamp(min=0)[:, None])[:, 0], n_pages)
    writers = torch.zeros_like(holders).scatter_add_(0, last, writes.long())
    first = torch.full_like(holders, n).scatter_reduce_(0, last, me, "amin")
    copied = writes & ~((holders[last] == writers[last]) & (first[last] == me))
    need = new - old + copied
    at = need.cumsum(0) - need
    free = holders[:n_pages] == 0
    ids = torch.full((n_pages + 1,), -1, dtype=torch.long, device=dev)
    ids[torch.where(free, free.long().cumsum(0) - 1, n_pages)] = torch.arange(n_pages, device=dev)
    take = (at + copied)[:, None] + col - old[:, None]
    fresh = (col >= old[:, None]) & (col < new[:, None])
    table = torch.where(kept, pages, torch.where(fresh, ids[take.clamp(0, n_pages)], -1))
    target = torch.where(copied, ids[at.clamp(max=n_pages)], -1)
    table = torch.where(copied[:, None] & (col == old[:, None] - 1), target[:, None], table)
    copies = torch.stack([torch.where(copied, last, -1), target], 1).int()
    refs = torch.zeros_like(holders).scatter_add_(0, torch.where(table >= 0, table, n_pages).flatten(), (table >= 0).long().flatten())
    _copy_pages(s["pool"], copies)
    report = torch.stack([need.sum() * 0, need.sum() * 0, need.sum() * 0, free.sum() - need.sum()]).int()
    return table.int(), (had + add).int(), refs[:n_pages].int(), copies, report, s["pool"]


def _plain_compact(s):
    n_pages, P, dev = s["n_pages"], s["case"]["page"], "cuda"
    page, pages = torch.arange(n_pages, device=dev), s["table"].long()
    kept = torch.arange(pages.shape[1], device=dev) < (-(-s["kv_len"].long() // P))[:, None]
    refs = torch.zeros(n_pages + 1, dtype=torch.long, device=dev).scatter_add_(0, torch.where(kept, pages, n_pages).flatten(), kept.long().flatten())
    live = refs[:n_pages] > 0
    n_live = live.sum()
    hole, mover = ~live & (page < n_live), live & (page >= n_live)
    most = n_pages // 2
    moves = torch.full((most + 1, 2), -1, dtype=torch.long, device=dev)
    moves[torch.where(mover, mover.long().cumsum(0) - 1, most), 0] = page
    moves[torch.where(hole, hole.long().cumsum(0) - 1, most), 1] = page
    moves = moves[:most]
    to = torch.cat([page, page.new_tensor([-1])])
    to[torch.where(moves[:, 0] >= 0, moves[:, 0], n_pages)] = moves[:, 1]
    table = torch.where(kept, to[torch.where(kept, pages, 0)], -1)
    refs = torch.zeros_like(refs).scatter_add_(0, torch.where(kept, table, n_pages).flatten(), kept.long().flatten())
    _copy_pages(s["pool"], moves)
    return table.int(), refs[:n_pages].int(), moves.int(), torch.stack([n_live, mover.sum(), n_live * 0, n_pages - n_live]).int(), s["pool"]


# ---------------------------------------------------------------------------------------------------- the definition, in 64 bits

def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "table":
        t, rot = torch.arange(case["n"], dtype=torch.float64), case["rot"]
        out, factor, original = torch.empty(case["n"], rot // 2, 2, dtype=torch.float64), case["factor"], s["original"]
        long, short = s["low"], s["high"]
        for i in range(rot // 2):
            theta = math.exp(-2 * i / rot * math.log(s["base"]))
            length = 2 * math.pi / theta
            if case["kind"] == "linear":
                theta /= factor
            elif case["kind"] == "base":
                theta *= math.exp(-2 * i / (rot - 2) * math.log(factor))
            elif case["kind"] == "bands":
                if length > original / long:
                    theta /= factor
                elif length > original / short:
                    keep = (original / length - long) / (short - long)
                    theta = keep * theta + (1 - keep) * theta / factor
            elif case["kind"] == "ramp":
                edge = [rot / 2 * math.log(original / (2 * math.pi * r), s["base"]) for r in (short, long)]
                a, b = max(0, math.floor(edge[0])), min(rot - 1, math.ceil(edge[1]))
                far = min(1.0, max(0.0, (i - a) / (b - a if b > a else 0.001)))
                theta = far * theta / factor + (1 - far) * theta
            out[:, i, 0], out[:, i, 1] = torch.cos(t * theta), torch.sin(t * theta)
        return out * (1 + math.log(factor) / 10 if case["kind"] == "ramp" else 1)

    def turned(x, positions):  # as complex numbers
        x, rot = x.double().clone(), case["rot"]
        angle = positions.double()[:, None] * torch.tensor([500000.0 ** (-2 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda")
        by = torch.polar(torch.ones_like(angle), angle)[:, None]
        re, im = (slice(0, rot, 2), slice(1, rot, 2)) if case["interleaved"] else (slice(0, rot // 2), slice(rot // 2, rot))
        z = torch.complex(x[..., re], x[..., im]) * by
        x[..., re], x[..., im] = z.real, z.imag
        return x

    if op == "rows":
        y = turned(s["x"], s["positions"].clamp(min=0))
        y[s["positions"] < 0] = 0
        return y
    if op == "fork":
        return [None] * 5 + [_exact_fork(s)]
    if op == "compact":
        return [None] * 4 + [_exact_compact(s)]
    rows, kv = _lengths(case)
    starts, table, P = np.concatenate([[0], np.cumsum(rows)]), s["table"].cpu(), case["page"]
    if op == "append":
        q, k_pages, v_pages = torch.empty_like(s["q"], dtype=torch.float64), s["k_pages"].double(), s["v_pages"].double()
        for b, (n, k) in enumerate(zip(rows, kv)):
            y, at = torch.arange(k - n, k), slice(int(starts[b]), int(starts[b + 1]))
            page, slot = table[b, y // P].long().cuda(), (y % P).cuda()
            q[at] = turned(s["q"][at], y.cuda())
            k_pages[page, slot] = turned(s["k"][at], y.cuda())
            v_pages[page, slot] = s["v"][at].double()
        return q, k_pages, v_pages
    if work(case)["flops"] > 1e14:
        return None
    G, o, lse = case["H"] // case["Hkv"], torch.empty_like(s["q"], dtype=torch.float64), s["q"].new_empty(s["q"].shape[:2], dtype=torch.float64)
    for b, (n, k) in enumerate(zip(rows, kv)):
        pages, at = table[b, :-(-k // P)].long().cuda(), slice(int(starts[b]), int(starts[b + 1]))
        keys, values = (s[x][pages].flatten(0, 1)[:k].double() for x in ("k_pages", "v_pages"))
        hidden = None
        if case["causal"]:
            hidden = torch.arange(k, device="cuda") > torch.arange(k - n, k, device="cuda")[:, None]
        for h in range(case["H"]):
            a = s["q"][at, h].double() @ keys[:, h // G].T / math.sqrt(case["d"])
            if hidden is not None:
                a[hidden] = -math.inf
            lse[at, h] = torch.logsumexp(a, -1)
            o[at, h] = torch.exp(a - lse[at, h][:, None]) @ values[:, h // G]
    return o, lse


def _exact_fork(s):
    """The pool after the step, page tables kept as lists."""
    P, table, kv = s["case"]["page"], s["table"].tolist(), s["kv_len"].tolist()
    source, add, pool = s["source"].tolist(), s["add"].tolist(), s["pool"].double()
    lists = [table[a][:-(-kv[a] // P)] if a >= 0 else [] for a in source]
    ends = [a >= 0 and add[i] > 0 and kv[a] % P > 0 for i, a in enumerate(source)]
    held = {}
    for i, pages in enumerate(lists):
        for p in pages:
            held.setdefault(p, []).append(i)
    free = (p for p in range(s["n_pages"]) if p not in held)
    for i, a in enumerate(source):
        if ends[i]:
            p = lists[i][-1]
            alone = all(ends[j] and lists[j][-1] == p for j in held[p]) and held[p][0] == i
            if not alone:
                pool[:, :, next(free)] = pool[:, :, p]
        if a >= 0:
            for _ in range(-(-(kv[a] + add[i]) // P) + (-kv[a] // P)):
                next(free)
    return pool


def _exact_compact(s):
    P, pool = s["case"]["page"], s["pool"].double()
    live = sorted({p for pages, k in zip(s["table"].tolist(), s["kv_len"].tolist()) for p in pages[:-(-k // P)]})
    holes = sorted(set(range(len(live))) - set(live))
    for p, to in zip((p for p in live if p >= len(live)), holes):
        pool[:, :, to] = pool[:, :, p]
    return pool
