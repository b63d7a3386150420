"""Rotary rows, scaled tables and the append to pages against 64 bits."""
import math

import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2507_05228_b200 import binding as cb

pytestmark = pytest.mark.gpu


def rows(n, H, d, dtype, seed=0):
    return torch.randn((n, H, d), generator=torch.Generator().manual_seed(seed)).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("n,H,d,rot", [(1, 1, 64, 64), (1, 32, 128, 128), (7, 5, 64, 16), (33, 12, 128, 96), (130, 3, 128, 32), (65, 8, 64, 48)])
def test_rows(dtype, interleaved, n, H, d, rot):
    x = rows(n, H, d, dtype, n)
    table = cb.cascade_rope_table(5000, rot, 10000.0)
    positions = torch.randint(0, 5000, (n,), generator=torch.Generator().manual_seed(1))
    positions[0] = 4999
    y = cb.cascade_rope_rows(x.cuda(), positions.int().cuda(), table, interleaved=interleaved)
    want = pu.turn(x, positions, table.cpu(), interleaved)
    off = pu.turn_bound(x, table.cpu(), positions, dtype, rot, interleaved)
    assert ((y.double().cpu() - want).abs() <= off).all()
    assert torch.equal(y.cpu()[..., rot:], x[..., rot:])
    place = x.cuda()
    assert cb.cascade_rope_rows(place, positions.int().cuda(), table, interleaved=interleaved, out=place) is place
    assert torch.equal(place, y)


def test_rows_agree_with_blocks():
    """The half layout on a block of consecutive positions is cascade_rope_apply."""
    x = rows(50, 4, 128, torch.bfloat16).cuda()
    table = cb.cascade_rope_table(100, 128, 10000.0)
    y = cb.cascade_rope_rows(x, torch.arange(20, 70, dtype=torch.int32, device="cuda"), table)
    assert torch.equal(y, cb.cascade_rope_apply(x[None], 20, table)[0])


def test_padded_bad_and_strided_rows():
    packed = rows(9, 7, 128, torch.bfloat16).cuda()
    x, table = packed[:, 2:5], cb.cascade_rope_table(10, 128, 10000.0)
    out = torch.full((9, 5, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    positions = [0, 9, -1, 10, 5, -2 ** 31, 2 ** 31 - 1, 2, 1]
    cb.cascade_rope_rows(x, pu.ints(positions), table, out=out[:, 1:4])
    with pytest.raises(cb.CascadeError, match="code 124"):
        cb.cascade_paged_status()
    good = torch.tensor([0, 1, 4, 7, 8])
    want = cb.cascade_rope_rows(x[good.cuda()].contiguous(), pu.ints([0, 9, 5, 2, 1]), table)
    assert torch.equal(out[good.cuda(), 1:4], want) and (out[[2, 3, 5, 6]] == 3).all() and (out[:, [0, 4]] == 3).all()
    assert cb.cascade_paged_status() == 0


@pytest.mark.parametrize("kind,rot,base,factor,original,low,high", [
    ("none", 128, 10000.0, 1.0, 0, 1, 4), ("linear", 64, 10000.0, 8.0, 0, 1, 4), ("base", 128, 10000.0, 4.0, 0, 1, 4),
    ("bands", 128, 500000.0, 8.0, 8192, 1, 4), ("bands", 2, 500000.0, 8.0, 8192, 1, 4), ("ramp", 128, 10000.0, 16.0, 4096, 1, 32),
    ("ramp", 64, 150000.0, 32.0, 4096, 1, 32), ("ramp", 16, 10.0, 2.0, 100, 1, 1.5)])
def test_scaled_table(kind, rot, base, factor, original, low, high):
    n = 4097
    got = cb.cascade_rope_table_scaled(n, rot, base, kind, factor, original, low, high).double().cpu().numpy()
    t, scale = np.arange(n, dtype=np.float64), 1.0
    for i in range(rot // 2):
        theta = base ** (-2 * i / rot)
        if kind == "linear":
            theta /= factor
        elif kind == "base":
            theta = (base * factor ** (rot / (rot - 2))) ** (-2 * i / rot)
        elif kind == "bands":
            turns = original * theta / (2 * math.pi)
            keep = 1.0 if turns >= high else 0.0 if turns <= low else (turns - low) / (high - low)
            theta = theta * keep + theta / factor * (1 - keep)
        elif kind == "ramp":
            scale = 0.1 * math.log(factor) + 1
            D = lambda turns: rot * math.log(original / (2 * math.pi * turns)) / (2 * math.log(base))  # noqa: E731
            a, b = max(0, math.floor(D(high))), min(rot - 1, math.ceil(D(low)))
            far = 0.0 if i <= a else 1.0 if i >= b else (i - a) / (b - a)
            theta = theta * (1 - far) + theta / factor * far
        # an angle of t theta in 64 bits is off by a few 2^-53 of itself, far below the rounding to fp32
        off = scale * (2.0 ** -24 + n * 2.0 ** -50)
        assert np.abs(got[:, i, 0] - scale * np.cos(t * theta)).max() <= off and np.abs(got[:, i, 1] - scale * np.sin(t * theta)).max() <= off


def test_scaled_table_without_scaling_is_the_table():
    assert torch.equal(cb.cascade_rope_table_scaled(777, 96, 500000.0), cb.cascade_rope_table(777, 96, 500000.0))
    twice = cb.cascade_rope_table_scaled(777, 96, 500000.0, "linear", 1.0, attention=2.0)
    assert torch.equal(twice, 2 * cb.cascade_rope_table(777, 96, 500000.0))


@pytest.mark.parametrize("dtype,d,rot", [(torch.bfloat16, 128, 128), (torch.bfloat16, 64, 32), (torch.float32, 64, 64), (torch.float32, 128, 16)])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("news,lens,page", [([1], [1], 16), ([1, 1, 1], [40, 1, 17], 16), ([0, 5, 0, 33, 1, 0], [7, 5, 0, 100, 65, 64], 48),
                                            ([1] * 70, list(range(1, 71)), 16), ([3] * 1100, [3 + i % 50 for i in range(1100)], 16)])
def test_append(dtype, d, rot, interleaved, news, lens, page):
    H, Hkv, lead, pad = 6, 2, 2, 3
    b = pu.Batch(news, lens, H, Hkv, d, page, dtype, seed=3, head_major=interleaved, lead=lead, pad=pad)
    k, v = rows(b.n, Hkv, d, dtype, 5), rows(b.n, Hkv, d, dtype, 6)
    table = cb.cascade_rope_table(200, rot, 10000.0)
    before = b.k_pages.clone(), b.v_pages.clone()
    q_out = torch.full_like(b.q, 9.0)
    cb.cascade_paged_append(k.cuda(), v.cuda(), b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, q=b.q, rope_table=table,
                            interleaved=interleaved, q_out=q_out)
    assert cb.cascade_paged_status() == 0
    want_k, want_v, off_k = before[0].double().cpu(), before[1].cpu(), torch.zeros(b.k_pages.shape, dtype=torch.float64)
    tab, t64 = b.table.cpu(), table.cpu()
    inside = torch.zeros(b.n, dtype=torch.bool)
    for s, (n, x) in enumerate(zip(news, lens)):
        r = slice(int(b.starts[s]), int(b.starts[s + 1]))
        inside[r] = True
        y = torch.arange(x - n, x)
        page_id, slot = tab[s, y // page].long(), y % page
        want_k[page_id, slot] = pu.turn(k[r], y, t64, interleaved)
        off_k[page_id, slot] = pu.turn_bound(k[r], t64, y, dtype, rot, interleaved)
        want_v[page_id, slot] = v[r]
        if n:
            off = pu.turn_bound(b.q64[r], t64, y, dtype, rot, interleaved)
            assert ((q_out[r].double().cpu() - pu.turn(b.q64[r], y, t64, interleaved)).abs() <= off).all()
    got = b.k_pages.double().cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want_k)) and ((got - want_k).abs() <= off_k)[~torch.isnan(got)].all()
    assert torch.equal(torch.nan_to_num(b.v_pages.cpu(), nan=77.0), torch.nan_to_num(want_v, nan=77.0))
    assert (q_out.cpu()[~inside] == 9).all()


def test_append_without_rotary_step_by_given_positions_and_in_place():
    b = pu.Batch([4, 2], [20, 33], 4, 2, 128, 16)
    k, v = rows(b.n, 2, 128, torch.bfloat16, 1).cuda(), rows(b.n, 2, 128, torch.bfloat16, 2).cuda()
    assert cb.cascade_paged_append(k, v, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len) is None
    page = b.table[1, 2].item()
    assert torch.equal(b.k_pages[page, 0], k[5]) and torch.equal(b.v_pages[page, 0], v[5])
    table = cb.cascade_rope_table(3000, 128, 10000.0)
    pos = pu.ints([7, 2999, 0, 12, 500, 501, 1, 2, 3])
    want = cb.cascade_rope_rows(b.q, pos, table), cb.cascade_rope_rows(k, pos, table)
    q = b.q.clone()
    assert cb.cascade_paged_append(k, v, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, q=q, positions=pos, rope_table=table, q_out=q) is q
    assert torch.equal(q[:6], want[0][:6]) and torch.equal(q[6:], b.q[6:])
    assert torch.equal(b.k_pages[page, 0], want[1][5]) and torch.equal(b.k_pages[b.table[0, 1].item(), 3], want[1][3])


@pytest.mark.parametrize("what", ["page", "length", "short", "rows", "position"])
def test_append_writes_nothing_where_an_index_is_bad(what):
    b = pu.Batch([4, 2], [20, 33], 4, 2, 64, 16)
    k, v = rows(b.n, 2, 64, torch.bfloat16, 1).cuda(), rows(b.n, 2, 64, torch.bfloat16, 2).cuda()
    table = cb.cascade_rope_table(40, 64, 10000.0)
    good = b.k_pages.clone(), b.v_pages.clone()
    cb.cascade_paged_append(k, v, good[0], good[1], b.table, b.row_start, b.kv_len, rope_table=table)
    pages = b.table[0].tolist()
    code, skipped = {"page": (123, [pages[1]]), "length": (122, None), "short": (122, None), "rows": (121, None), "position": (124, None)}[what]
    pos = None
    if what == "page":
        b.table[0, 1] = b.n_pages  # rows 16 .. 19 of the first sequence
    elif what == "length":
        b.kv_len[0] = -3
    elif what == "short":
        b.kv_len[0] = 3  # fewer rows than are new: the first has no place
    elif what == "rows":
        b.row_start[1] = 100
    else:
        pos = pu.ints([40] * 4 + [31, 32] + [0] * 3)
    before = b.k_pages.clone(), b.v_pages.clone()
    cb.cascade_paged_append(k, v, b.k_pages, b.v_pages, b.table, b.row_start, b.kv_len, positions=pos, rope_table=table)
    with pytest.raises(cb.CascadeError, match=f"code {code}"):
        cb.cascade_paged_status()
    assert cb.cascade_paged_status() == 0
    changed = [i for i in range(b.n_pages) if not torch.equal(torch.nan_to_num(b.k_pages[i].float()), torch.nan_to_num(before[0][i].float()))]
    second = b.table[1, 1:3].tolist() if what != "rows" else []
    if what == "page":
        assert sorted(changed) == sorted(second)
    elif what == "short":  # the three that have a place
        assert sorted(changed) == sorted(second + [pages[0]])
    else:
        assert sorted(changed) == sorted(second) or what == "rows"


def test_append_beyond_32_bits_of_offset():
    page, Hkv, d = 16, 8, 128
    n_pages = 2 ** 31 // (page * Hkv * d) + 300  # elements past 2^31
    k_pages, v_pages = (torch.zeros((n_pages, page, Hkv, d), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k, v = rows(1, Hkv, d, torch.bfloat16, 1).cuda(), rows(1, Hkv, d, torch.bfloat16, 2).cuda()
    cb.cascade_paged_append(k, v, k_pages, v_pages, pu.ints([[3, n_pages - 1]]), pu.ints([0, 1]), pu.ints([20]))
    assert torch.equal(k_pages[n_pages - 1, 3], k[0]) and torch.equal(v_pages[n_pages - 1, 3], v[0])
    assert k_pages.count_nonzero() == k.count_nonzero()
