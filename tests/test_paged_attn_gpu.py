"""cascade_attn_paged against 64 bits: ragged rows, lengths from none on, pages that end inside a tile, masks that leave rows empty."""
import math

import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2507_05228_b200 import binding as cb

pytestmark = pytest.mark.gpu


def attend(b, causal=True, visible=None, max_rows=None, **more):
    out = torch.full((b.n, b.H, b.d), 5.0, dtype=b.dtype, device="cuda")
    before = out.clone()
    o, lse = cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, causal=causal,
                                   visible=None if visible is None else pu.ints(visible), max_rows=max_rows, out=out, **more)
    assert o is out and cb.cascade_paged_status() == 0
    b.check(out, lse, causal, visible, before)
    return out, lse


TYPES = [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64), (torch.float32, 128)]
HEADS = [(1, 1), (8, 2), (12, 12), (8, 1), (6, 2), (32, 2)]


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("page", [16, 48, 256])
def test_single_tokens(dtype, d, H, Hkv, page):
    lens = [1, 15, 16, 17, 0, 33, 127, 128, 129, 700, 5]
    b = pu.Batch([1] * len(lens), lens, H, Hkv, d, page, dtype, seed=H + page)
    attend(b, max_rows=1)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("n", [2, 7, 37, 100])
def test_tokens_and_drafts_behind_wide_tables(dtype, d, H, Hkv, n):
    """Tables with room for 64000 rows, which nobody has: how the keys are shared out goes by the lengths on the device.  One sequence
    is far longer than the others, some are empty, some have no new row, and the rows of the others are one to four."""
    rng = np.random.default_rng(n + H)
    lens = [int(x) for x in rng.integers(0, 90, n)]
    lens[n // 2], lens[-1] = 1500 if H < 32 else 700, 0
    news = [int(x) for x in rng.integers(1, 1 + max(1, min(4, 16 * Hkv // H)), n)]
    if n > 3:
        news[1] = 0
    b = pu.Batch(news, lens, H, Hkv, d, 32, dtype, seed=n, width=2000)
    attend(b, max_rows=4)
    attend(b, causal=False, max_rows=4)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("H,Hkv", HEADS)
@pytest.mark.parametrize("causal", [True, False])
def test_chunks_of_any_size(dtype, d, H, Hkv, causal):
    """Tokens, drafts, chunks and whole prompts side by side; sequences without new rows, without a cache, and with more new rows than
    the cache has (the first of which see nothing)."""
    news, lens = [1, 0, 3, 130, 64, 20, 2, 9, 257, 0], [50, 40, 3, 131, 300, 17, 0, 5, 257, 0]
    b = pu.Batch(news, lens, H, Hkv, d, 16 if causal else 64, dtype, seed=H, lead=2, head_major=not causal, strided=causal)
    attend(b, causal=causal)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("page", [16, 32, 48, 64, 80, 112, 128, 144, 256])
def test_page_sizes(dtype, d, page):
    for news, lens in (([200], [1000]), ([5, 1, 2], [500, 333, 90])):
        attend(pu.Batch(news, lens, 4, 1, d, page, dtype, seed=page))


@pytest.mark.parametrize("dtype,d", TYPES)
def test_lengths_around_tiles(dtype, d):
    for n in (1, 2, 16, 17, 31, 33, 63, 65, 128, 129):
        lens = [n, n + 1, 127, 128, 129, 256 + n]
        lens = [max(x, n) for x in lens]
        attend(pu.Batch([n] * 6, lens, 4, 2, d, 32, dtype, seed=n), max_rows=n)


@pytest.mark.parametrize("dtype,d", TYPES)
@pytest.mark.parametrize("news", [[1, 1, 1, 1], [70, 3, 200, 1]])
def test_prefixes_given_by_row(dtype, d, news):
    """Any prefix, in any order of the rows, none and more than there is among them."""
    lens = [300, 40, 513, 64]
    b = pu.Batch(news, lens, 8, 2, d, 16, dtype, seed=4)
    rng = np.random.default_rng(7)
    visible = rng.integers(-2, 400, b.n)
    visible[0], visible[-4] = 0, 10 ** 6
    attend(b, visible=visible)
    attend(b, visible=np.zeros(b.n, int))


@pytest.mark.parametrize("dtype,d", TYPES)
def test_rows_that_one_key_dominates(dtype, d):
    """Long keys: weights of one for one key, and logits that rise by hundreds from one tile to the next."""
    for news in ([1, 1], [100, 33]):
        b = pu.Batch(news, [400, 290], 4, 2, d, 32, dtype, seed=2, scale_k=30.0)
        attend(b)


def test_logits_of_minus_infinity_and_the_lowest_value():
    """Keys whose logits overflow to -inf carry no weight; a row of nothing else yields zeros."""
    for dtype, news in ((torch.bfloat16, [1]), (torch.bfloat16, [40]), (torch.float32, [1]), (torch.float32, [40])):
        b = pu.Batch(news, [200], 2, 2, 64, 16, dtype, seed=8)
        b.q[:, 0] = 1.0
        b.q64[:, 0] = 1.0
        b.k_rows[0][:150, 0] = -1.0
        big = torch.finfo(dtype).min / 2
        pages = b.table[0].cpu()
        for y in range(150):
            b.k_pages[pages[y // 16].item(), y % 16, 0] = big
        out, lse = cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, causal=False)
        assert torch.isfinite(out[:news[0]].float()).all()
        b.k_rows[0][:150, 0] = -1e30
        b.lens[0] = 200
        o_ref, lse_ref, _, _ = b.reference(causal=False)
        assert (out[:news[0]].double().cpu() - o_ref[:news[0]]).abs().max() < 0.03 and (lse[:news[0]].double().cpu() - lse_ref[:news[0]]).abs().max() < 1e-3


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,Hkv", [(1, 1), (12, 12), (4, 2), (6, 2), (8, 2), (14, 2), (8, 1), (24, 2), (32, 2)])
@pytest.mark.parametrize("n", [1, 2, 5, 60])
def test_drafts_of_every_width(d, H, Hkv, n):
    """Up to 32 (row, head) pairs of a KV head, and one row more: one sequence, a few over short and over wide tables, many; lengths that
    end inside a block of 16 and inside a page, and caches shorter than the drafts."""
    group, rng = H // Hkv, np.random.default_rng(100 * n + H)
    for pairs in (9, 16, 17, 24, 25, 32):
        rows = max(1, min(pairs, 32) // group)
        news = [rows] + [int(x) for x in rng.integers(0, rows + 1, n - 1)]
        lens = [int(x) for x in rng.integers(0, 500, n)]
        lens[0], lens[-1] = 16 * 23 + 1 + pairs % 16, max(1, rows - 1)
        strided = pairs == 16
        for width in ([0, 2000] if n > 1 else [0]):
            b = pu.Batch(news, lens, H, Hkv, d, 48 if pairs == 24 else 16 if pairs == 32 else 64, seed=pairs, head_major=pairs == 25, strided=strided,
                         **({"width": width} if width else {}))
            attend(b, max_rows=rows)
            if width == 0 and pairs in (17, 32):
                attend(b, causal=False, max_rows=rows + 1)
                attend(b, visible=rng.integers(-3, 600, b.n), max_rows=rows)


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,Hkv", [(5, 1), (7, 1), (8, 1), (16, 1), (24, 2), (28, 4), (40, 2)])
@pytest.mark.parametrize("n", [1, 2, 6])
def test_drafts_whose_heads_are_split(d, H, Hkv, n):
    """More (row, head) pairs than a KV head's columns, few sequences: its heads go to several parts of the chip."""
    for rows in (3, 5, 8):
        lens = [700, 0, 33, 2500, 7, 160][:n]
        news = [rows, 0, rows - 1, 1, rows, 2][:n]
        for width in ([0, 900] if n > 1 else [0]):
            b = pu.Batch(news, lens, H, Hkv, d, 32, seed=rows, **({"width": width} if width else {}))
            attend(b, max_rows=rows)
            attend(b, causal=False, max_rows=rows)


@pytest.mark.parametrize("n", [3, 12, 40])
@pytest.mark.parametrize("width", [0, 300])
def test_captured_drafts_side_by_side(n, width):
    """Two graphs with a workspace each, replayed on two streams over lengths that have changed: a CTA an item, shares, ranges."""
    full = [300 + 37 * i % 600 for i in range(n)]
    b = pu.Batch([1 + i % 6 for i in range(n)], full, 16, 4, 128, 32, seed=n, **({"width": width} if width else {}))
    runs = []
    for _ in range(2):
        out, stream, graph = torch.zeros_like(b.q), torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for _ in range(3):
                _, lse = cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, max_rows=6, out=out)
        runs.append((graph, stream, out, lse))
    k_rows, v_rows = b.k_rows, b.v_rows
    for cut in (0, 250, 290):
        lens = [x - cut for x in full]
        b.kv_len.copy_(pu.ints(lens))
        b.lens, b.k_rows, b.v_rows = lens, [k[:x] for k, x in zip(k_rows, lens)], [v[:x] for v, x in zip(v_rows, lens)]
        torch.cuda.synchronize()
        for graph, stream, _, _ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        for _, _, out, lse in runs:
            b.check(out, lse)
    assert cb.cascade_paged_status() == 0


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,Hkv", [(2, 2), (4, 1), (8, 1), (12, 2)])
@pytest.mark.parametrize("n", [1, 3])
def test_chunks_that_fill_one_sub_tile(d, H, Hkv, n):
    """At most 128 (row, head) pairs a KV head: tiles of keys from one to many, an odd number of them, shared by clusters or not."""
    group = H // Hkv
    group = 2 if group == 6 else group  # heads that are stacked: a power of two
    for pairs in (40, 100, 128):
        rows = pairs // group
        for lens in ([rows + 1, 128, 129], [257, 0, 300], [1500, 640, 641], [2999, 33, 385]):
            news = [rows, max(1, rows - 7), rows]
            b = pu.Batch(news[:n], lens[:n], H, Hkv, d, 32, seed=pairs, scale_k=8.0 if pairs == 100 else 1.0)
            attend(b, max_rows=rows)
            attend(b, causal=False, max_rows=rows)
            attend(b, visible=np.random.default_rng(pairs).integers(-2, 3200, b.n), max_rows=rows)


@pytest.mark.parametrize("d", [128, 64])
def test_more_rows_than_announced_in_a_sub_tile(d):
    """max_rows chooses kernels and nothing else on tiles: a sequence with more rows than it says is right all the same."""
    b = pu.Batch([200, 40, 64], [700, 300, 64], 4, 2, d, 32, seed=3)
    attend(b, max_rows=64)


def test_long_cache_and_many_sequences():
    attend(pu.Batch([1, 4], [20001, 9000], 8, 2, 128, 64, seed=1), max_rows=4)
    attend(pu.Batch([1] * 300, [1 + 7 * i % 200 for i in range(300)], 4, 2, 64, 16, seed=2), max_rows=1)
    attend(pu.Batch([i % 5 for i in range(400)], [4 + i % 90 for i in range(400)], 4, 1, 128, 16, seed=3), max_rows=4)


def test_pool_beyond_32_bits_of_offset():
    b = pu.Batch([1, 30], [100, 200], 8, 2, 128, 16, seed=1)
    n_pages = 2 ** 31 // (16 * 2 * 128) + b.n_pages
    for name in ("k_pages", "v_pages"):
        small = getattr(b, name)
        big = torch.empty((n_pages,) + small.shape[1:], dtype=b.dtype, device="cuda")
        big[n_pages - b.n_pages:] = small
        setattr(b, name, big)
    used = (b.table >= 0) & (b.table < b.n_pages)
    b.table = torch.where(used, b.table + (n_pages - b.n_pages), b.table)
    attend(b)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("news", [[1, 1, 2], [1, 90, 300]])
def test_bad_indices_are_reported_and_the_other_sequences_right(dtype, news):
    for what, code in (("page", 123), ("negative", 123), ("length", 122), ("long", 122), ("rows", 121)):
        b = pu.Batch(news, [100, 200, 300], 4, 2, 128, 16, dtype, seed=1)
        torch.nan_to_num_(b.k_pages)  # (a page that is read by mistake holds finite values)
        torch.nan_to_num_(b.v_pages)
        if what == "page":
            b.table[1, 3] = b.n_pages
        elif what == "negative":
            b.table[1, 3] = -1
        elif what == "length":
            b.kv_len[1] = -1
        elif what == "long":
            b.kv_len[1] = b.table.shape[1] * 16 + 1
        else:
            b.row_start[3] = b.n + 1  # the last sequence
        got = cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale)[0]
        with pytest.raises(cb.CascadeError, match=f"code {code}"):
            cb.cascade_paged_status()
        assert cb.cascade_paged_status() == 0
        o_ref, _, off, _ = b.reference()  # of the sequences as they were
        others = [0, 2] if what != "rows" else [0, 1]
        for s in others:
            r = slice(int(b.starts[s]), int(b.starts[s + 1]))
            assert ((got[r].double().cpu() - o_ref[r]).abs() <= off[r]).all(), (what, s)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("news", [[1, 1, 1], [1, 100, 20]])
def test_captured_calls_follow_their_lengths(dtype, news):
    """Two graphs of the same call, with a workspace each, replayed side by side on two streams over lengths that have changed."""
    b = pu.Batch(news, [700, 400, 310], 8, 2, 128, 16, dtype, seed=6)
    full = list(b.lens)
    L = cb.lib()
    runs = []
    for _ in range(2):
        out = torch.zeros_like(b.q)
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, out=out)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            _, lse = cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, out=out)
        runs.append((graph, stream, out, lse))
    for lens in ([700, 400, 310], [129, 100, 20], [1, 333, 200]):
        lens = [min(x, f) for x, f in zip(lens, full)]
        b.kv_len.copy_(pu.ints(lens))
        torch.cuda.synchronize()
        n0 = L.cascade_launch_count()
        for graph, stream, out, _ in runs:
            with torch.cuda.stream(stream):
                graph.replay()
        torch.cuda.synchronize()
        assert L.cascade_launch_count() == n0
        b.lens = lens
        k_rows, v_rows = b.k_rows, b.v_rows
        b.k_rows, b.v_rows = [k[:x] for k, x in zip(k_rows, lens)], [v[:x] for v, x in zip(v_rows, lens)]
        for _, _, out, lse in runs:
            b.check(out, lse)
        b.k_rows, b.v_rows = k_rows, v_rows
    assert cb.cascade_paged_status() == 0


def test_the_same_call_gives_the_same_bits():
    for news in ([1] * 9, [1, 300, 5, 40]):
        b = pu.Batch(news, [900 + 31 * i for i in range(len(news))], 8, 2, 128, 64, seed=1)
        args = (b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale)
        o, lse = cb.cascade_attn_paged(*args)
        for _ in range(5):
            o2, lse2 = cb.cascade_attn_paged(*args, workspace=torch.randint(0, 255, (1 << 26,), dtype=torch.uint8, device="cuda"))
            assert torch.equal(o[:sum(news)], o2[:sum(news)]) and torch.equal(lse[:sum(news)], lse2[:sum(news)])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("news", [[1, 2, 1], [1, 90, 300]])
def test_layers_of_one_pool_and_strided_outputs(dtype, news):
    """Pages of K and V of several layers in one tensor, a table that is part of a wider one, outputs and queries inside wider rows."""
    b = pu.Batch(news, [100, 200, 310], 8, 2, 128, 16, dtype, seed=9, strided=True)
    pool = torch.full((b.n_pages, 3, 2, 16, 2, 128), math.nan, dtype=dtype, device="cuda")
    pool[:, 1, 0], pool[:, 1, 1] = b.k_pages, b.v_pages
    b.k_pages, b.v_pages = pool[:, 1, 0], pool[:, 1, 1]
    table = torch.full((3, 100), -5, dtype=torch.int32, device="cuda")
    table[:, 20:20 + b.table.shape[1]] = b.table
    b.table = table[:, 20:20 + b.table.shape[1]]
    wide = torch.full((b.n, 12, 160), 7.0, dtype=dtype, device="cuda")
    out = wide[:, 2:10, 16:144]
    o, lse = cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, out=out)
    assert cb.cascade_paged_status() == 0
    b.check(o, lse)
    wide[:, 2:10, 16:144] = 7.0
    assert (wide[:sum(news)] == 7).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("H,Hkv", [(21, 3), (20, 1), (34, 2), (64, 1)])
def test_odd_groups_of_heads(dtype, H, Hkv):
    for news, lens in (([1, 1, 2], [70, 33, 129]), ([40, 1, 3], [140, 33, 129])):
        attend(pu.Batch(news, lens, H, Hkv, 64, 16, dtype, seed=H))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("n,width", [(3, None), (3, 2000), (200, 2000)])
def test_more_rows_than_announced_are_reported_and_left(dtype, n, width):
    news = [1] * n
    news[1] = 3
    b = pu.Batch(news, [50 + i % 7 for i in range(n)], 8, 2, 64, 16, dtype, seed=1, width=width)
    out = torch.full((b.n, 8, 64), 5.0, dtype=dtype, device="cuda")
    cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, max_rows=1, out=out)
    with pytest.raises(cb.CascadeError, match="code 126.*sequence 1, value 3"):
        cb.cascade_paged_status()
    o_ref, _, off, _ = b.reference()
    others = [r for r in range(sum(news)) if r not in (1, 2, 3)]
    assert ((out.double().cpu() - o_ref).abs() <= off)[others].all() and (out[1:4] == 5).all()


def test_calls_on_several_streams_at_once():
    """Chunks, tokens and fp32 side by side, again and again, each with its own outputs and workspace."""
    cases = [pu.Batch([1] * 5, [300, 20, 900, 64, 1], 8, 2, 128, 16, seed=1), pu.Batch([70, 1, 200], [300, 20, 900], 8, 2, 128, 16, seed=2),
             pu.Batch([3, 60], [300, 200], 8, 2, 64, 16, torch.float32, seed=3), pu.Batch([1, 1], [3000, 2000], 8, 2, 64, 32, seed=4, width=2000)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    got = [[] for _ in cases]
    for _ in range(10):
        for b, s, g in zip(cases, streams, got):
            with torch.cuda.stream(s):
                g.append(cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale))
    torch.cuda.synchronize()
    assert cb.cascade_paged_status() == 0
    for b, g in zip(cases, got):
        b.check(*g[0])
        n = sum(b.rows)
        assert all(torch.equal(o[:n], g[0][0][:n]) and torch.equal(lse[:n], g[0][1][:n]) for o, lse in g[1:])


def test_no_rows():
    b = pu.Batch([2], [3], 4, 2, 64, 16)
    o, lse = cb.cascade_attn_paged(b.q[:0], b.k_pages, b.v_pages, b.table[:0], b.row_start[:1], b.kv_len[:0], b.scale)
    assert o.shape == (0, 4, 64) and lse.shape == (0, 4)


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.float32, 64)])
@pytest.mark.parametrize("n_q,offset", [(1, 299), (37, 200)])
def test_parties_with_pools_of_their_own(dtype, d, n_q, offset):
    """Each party keeps the rows of one KV shard in pages; its rows see what VIS of its plan says; (o, lse, 1) of all parties through
    cascade_merge is the attention over the whole cache."""
    n, H, Hkv, P, page = 300, 8, 2, 3, 16
    whole = pu.Batch([n_q], [offset + n_q], H, Hkv, d, page, dtype, seed=3, pad=0)
    shard = np.random.default_rng(1).integers(0, P, n)
    parts = []
    for k in range(P):
        held = np.flatnonzero(shard == k)
        plan = cb.cascade_shard_plan_resident(np.zeros(n_q, np.int32), np.zeros(held.size, np.int32), held.astype(np.int32), 1, 1, offset)
        vis = plan.get("vis")[0, :, 0]
        assert np.array_equal(vis, [(held <= offset + i).sum() for i in range(n_q)])
        mine = pu.Batch([n_q], [held.size], H, Hkv, d, page, dtype, seed=50 + k, pad=0)
        table = mine.table[0].tolist()
        rows_k, rows_v = torch.zeros(n, Hkv, d, dtype=dtype), torch.zeros(n, Hkv, d, dtype=dtype)
        rows_k[:offset + n_q], rows_v[:offset + n_q] = whole.k_rows[0].to(dtype), whole.v_rows[0].to(dtype)
        for y, t in enumerate(held):
            mine.k_pages[table[y // page], y % page] = rows_k[t].cuda()
            mine.v_pages[table[y // page], y % page] = rows_v[t].cuda()
        parts.append(cb.cascade_attn_paged(whole.q, mine.k_pages, mine.v_pages, mine.table, mine.row_start, mine.kv_len, whole.scale,
                                           visible=torch.from_numpy(vis.copy()).cuda()))
        plan.destroy()
    u, m = torch.stack([p[0] for p in parts])[None], torch.stack([p[1] for p in parts])[None]
    o, lse = cb.cascade_merge(u, m, torch.ones_like(m))
    o_ref, lse_ref, off_o, off_lse = whole.reference()
    # every part is rounded to the type once more, and weighs what it weighs: half a step of sum w |o_part| <= sum w |v|
    w_abs = off_o / (2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -21)
    assert ((o[0].double().cpu() - o_ref).abs() <= off_o + 1.01 * pu.HALF[dtype] * w_abs).all()
    assert ((lse[0].double().cpu() - lse_ref).abs() <= 3 * off_lse).all()
    assert cb.cascade_paged_status() == 0


def test_tensors_that_do_not_fit_are_refused():
    b = pu.Batch([2, 1], [30, 40], 4, 2, 64, 16)
    args = dict(q=b.q, k_pages=b.k_pages, v_pages=b.v_pages, page_table=b.table, row_start=b.row_start, kv_len=b.kv_len, scale=b.scale)
    for name, value in (("q", b.q.float()), ("q", b.q[..., :32]), ("v_pages", b.v_pages[:-1]), ("v_pages", b.v_pages.float()),
                        ("page_table", b.table.long()), ("page_table", b.table.T.contiguous().T), ("row_start", b.row_start[:2]), ("row_start", b.row_start.long()),
                        ("kv_len", b.kv_len[:1]), ("visible", b.kv_len), ("out", b.q[:2]), ("out", b.q.float())):
        with pytest.raises(ValueError):
            cb.cascade_attn_paged(**{**args, name: value})
    with pytest.raises(AssertionError):
        cb.cascade_attn_paged(**{**args, "q": b.q.transpose(1, 2)})
    with pytest.raises(cb.CascadeError, match="multiple"):
        cb.cascade_attn_paged(**{**args, "q": b.q[:, :3]})
    with pytest.raises(cb.CascadeError, match="page_size"):
        cb.cascade_attn_paged(**{**args, "k_pages": b.k_pages[:, :8], "v_pages": b.v_pages[:, :8]})
    if torch.cuda.device_count() > 1:
        with torch.cuda.device(1), pytest.raises(ValueError, match="device"):
            cb.cascade_attn_paged(**args)
    attend(b)
