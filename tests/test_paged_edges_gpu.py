"""Calls on paged caches that lie between the ordinary ones, against 64 bits."""
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


@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("H,Hkv,tokens", [(32, 8, 199), (32, 8, 200), (8, 2, 700), (8, 2, 701)])
@pytest.mark.parametrize("chunk,max_rows", [(300, None), (300, 300), (30, 30)])
def test_a_chunk_beside_many_single_tokens(d, H, Hkv, tokens, chunk, max_rows):
    """Few tiles there must be and many there could be, behind tables wide enough that the keys of a tile are shared by a cluster: an
    even and an odd number of tiles that could be; chunks of two sub-tiles and of one."""
    rng = np.random.default_rng(tokens + chunk)
    lens = [int(x) for x in rng.integers(0, 70, tokens)] + [900 + chunk]
    news = [1] * tokens + [chunk]
    place = tokens // 3
    lens[place], lens[-1], news[place], news[-1] = lens[-1], lens[place], news[-1], news[place]
    attend(pu.Batch(news, lens, H, Hkv, d, 32, seed=d + chunk, width=200), max_rows=max_rows)


@pytest.mark.parametrize("n", [1, 4])
@pytest.mark.parametrize("over", [1, 40])
def test_append_past_the_end_of_the_table_writes_nothing(n, over):
    """A sequence that has grown past its row of the table: its new rows have no place, and the last ones that do are another's."""
    b = pu.Batch([n, 2], [32, 20], 4, 2, 64, 16)
    k, v = (torch.randn((b.n, 2, 64), device="cuda").to(torch.bfloat16) for _ in range(2))
    b.table = b.table[:, :2].contiguous()
    b.kv_len[0] = 32 + over
    before = b.k_pages.clone(), b.v_pages.clone()
    q_out = torch.full_like(b.q, 9.0)
    cb.cascade_paged_append(k, v, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, q=b.q, q_out=q_out)
    with pytest.raises(cb.CascadeError, match=f"code 122.*sequence 0, value {32 + over}"):
        cb.cascade_paged_status()
    for pages, was in zip((b.k_pages, b.v_pages), before):
        for page in b.table[0].tolist():
            assert torch.equal(torch.nan_to_num(pages[page], nan=77.0), torch.nan_to_num(was[page], nan=77.0))
    page = b.table[1, 1].item()
    assert torch.equal(b.k_pages[page, 2:4], k[n:n + 2]) and torch.equal(b.v_pages[page, 2:4], v[n:n + 2])
    assert (q_out[:n] == 9).all() and torch.equal(q_out[n:n + 2], b.q[n:n + 2])


def poison(b, bits_of):
    """Elements of queries of some rows and heads by their bits; returns where (rows, heads)."""
    bad = torch.zeros(b.n, b.H, dtype=torch.bool)
    bits = b.q.view(torch.int32 if b.dtype == torch.float32 else torch.int16)
    for i, row in enumerate(sorted({0, b.n - 4, (b.n - 4) // 2, (b.n - 4) // 3})):
        bits[row, 3 * i % b.H, 7 * i % b.d] = bits_of[i]
        bad[row, 3 * i % b.H] = True
    return bad


def shows_in_its_row_alone(b, bad, max_rows):
    o_ref, lse_ref, off_o, off_lse = b.reference()  # of the queries as they were
    o, lse = cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, max_rows=max_rows)
    assert cb.cascade_paged_status() == 0
    o, lse = o.cpu(), lse.cpu()
    assert torch.isnan(o[bad]).all() and torch.isnan(lse[bad]).all()
    fine = ~bad
    fine[sum(b.rows):] = False
    assert ((o.double() - o_ref).abs() <= off_o)[fine].all() and ((lse.double() - lse_ref).abs() <= off_lse)[fine].all()


ROUTES = [([1] * 4, None), ([1] * 12, 2000), ([1] * 40, 2000), ([1] * 100, None), ([4, 1, 3, 2], None), ([4] * 12, 2000), ([6] * 30, 2000),
          ([30] * 3, None), ([30, 25], 200), ([70, 3, 200, 1], None), ([130], 200)]


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64), (torch.float32, 128)])
@pytest.mark.parametrize("news,width", ROUTES)
def test_a_query_that_is_not_a_number_shows_in_its_row_alone(dtype, d, news, width):
    """It is not a row that sees nothing, whose zeros and lse of -inf a merge would leave out."""
    rng = np.random.default_rng(len(news) + d)
    b = pu.Batch(news, [int(x) for x in rng.integers(200, 500, len(news))], 8, 2, d, 32, dtype, seed=5, width=width)
    bad = poison(b, [0x7fc00000] * 4 if dtype == torch.float32 else [0x7fff, -1, 0x7fc0, 0x7f81])
    shows_in_its_row_alone(b, bad, max(news))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("news,width", ROUTES)
def test_every_not_a_number_of_an_fp32_query_counts(d, news, width):
    """Those that arithmetic on the GPU makes among them, whose bits are all ones, and infinities."""
    rng = np.random.default_rng(len(news) + d)
    for bits in ([0x7fffffff, -1, 0x7fc00000, 0x7f800001], [0x7f800000, 0x7fffefff, 0x7ffff000, -0x800000]):
        b = pu.Batch(news, [int(x) for x in rng.integers(200, 500, len(news))], 8, 2, d, 32, torch.float32, seed=5, width=width)
        shows_in_its_row_alone(b, poison(b, bits), max(news))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("news", [[1], [1] * 12, [5, 40], [100]])
def test_the_largest_finite_queries_in_fp32(d, news):
    """A query of the type's largest value times keys that bring the logit back to ordinary size."""
    b = pu.Batch(news, [150 + i for i in range(len(news))], 4, 2, d, 32, torch.float32, seed=6)
    largest = torch.finfo(torch.float32).max
    b.q[:, 1] = 0
    b.q[:, 1, 5] = largest
    b.q64[:, 1] = 0
    b.q64[:, 1, 5] = largest
    table = b.table.cpu()
    for s, x in enumerate(b.lens):
        for y in range(x):
            small = (1 + y % 8) * 2.0 ** -125
            b.k_pages[table[s, y // 32].item(), y % 32, 0, 5] = small
            b.k_rows[s][y, 0, 5] = small
    attend(b)


def spoil_unseen(b, visible):
    """NaN in the K and V rows of the caches that no row of their sequence sees, though the length reaches them."""
    table = b.table.cpu()
    for s in range(len(b.rows)):
        seen = b.seen(s, True, visible)
        for y in range(int(max(seen, default=0)), b.lens[s]):
            b.k_pages[table[s, y // b.page].item(), y % b.page] = math.nan
            b.v_pages[table[s, y // b.page].item(), y % b.page] = math.nan


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64), (torch.float32, 128)])
@pytest.mark.parametrize("news,width", [([1] * 4, None), ([1] * 12, 2000), ([1] * 40, 2000), ([1] * 100, None), ([4, 1, 3, 2], None), ([8, 5, 1], None),
                                        ([4] * 12, 2000), ([6] * 30, 2000), ([3] * 90, None), ([30] * 3, None), ([30, 25], 200), ([70, 3, 200, 1], None),
                                        ([130], 200), ([33, 40], 200)])
def test_rows_of_the_cache_that_a_prefix_leaves_unseen_may_hold_anything(dtype, d, news, width):
    rng = np.random.default_rng(len(news) + d)
    lens = [int(x) for x in rng.integers(30, 400 if len(news) < 40 else 200, len(news))]
    b = pu.Batch(news, lens, 8, 2, d, 32, dtype, seed=4, width=width)
    visible = np.full(b.n, 5)
    for s in range(len(news)):
        most = [0, lens[s] // 3, lens[s] - 1, lens[s]][rng.integers(0, 4)]
        visible[b.starts[s]:b.starts[s + 1]] = rng.integers(0, most + 1, news[s])
    spoil_unseen(b, visible)
    attend(b, visible=visible, max_rows=max(news))


def test_max_rows_is_a_32_bit_number():
    b = pu.Batch([2, 1], [30, 40], 4, 2, 64, 16)
    for value in (2 ** 32 + 1, 2 ** 31, -2 ** 40):
        with pytest.raises(ValueError, match="max_rows"):
            cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, max_rows=value)
    attend(b, max_rows=2 ** 31 - 1)


def test_a_workspace_is_no_longer_than_its_memory():
    """A view that shows the same bytes again and again."""
    b = pu.Batch([1] * 40, [300] * 40, 8, 2, 64, 16, width=2000)
    small = torch.zeros(256, dtype=torch.uint8, device="cuda")
    for view in (small[:1].expand(1 << 26), small.expand(1 << 18, 256), small[:0]):
        with pytest.raises(cb.CascadeError, match="workspace"):
            cb.cascade_attn_paged(b.q, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, b.scale, max_rows=1, workspace=view)
    attend(b, max_rows=1, workspace=torch.zeros((1 << 13, 2 << 13), dtype=torch.uint8, device="cuda")[:, ::2])


@pytest.mark.parametrize("dtype,d", [(torch.bfloat16, 128), (torch.bfloat16, 64), (torch.float32, 64)])
@pytest.mark.parametrize("where", ["front", "ends", "spread"])
@pytest.mark.parametrize("places,rows", [(70, 1), (3000, 1), (3000, 4), (8192, 1), (70, 20), (3000, 20)])
def test_a_batch_of_idle_places(dtype, d, where, places, rows):
    """Places of a cache that nobody has taken: no rows and no length."""
    live = 50
    at = {"front": list(range(live)), "ends": list(range(live // 2)) + list(range(places - live // 2, places)),
          "spread": [i * (places - 1) // (live - 1) for i in range(live)]}[where]
    rng = np.random.default_rng(places)
    news, lens = [0] * places, [0] * places
    for i in at:
        news[i], lens[i] = int(rng.integers(1, rows + 1)), int(rng.integers(rows, 400))
    b = pu.Batch(news, lens, 8, 2, d, 16, dtype, seed=rows, width=200)
    attend(b, max_rows=rows)
