"""What the paged calls refuse on the host, before any CUDA call (no GPU needed)."""
import ctypes

import pytest
import torch

from paper_2507_05228_b200 import binding as cb

P = 4096  # stands for an aligned device address: nothing is launched


@pytest.fixture(scope="module")
def L():
    from paper_2507_05228_b200 import build
    build.build_library()
    return cb.lib()


def changed(args, **by_place):
    a = list(args)
    for place, value in by_place.items():
        a[int(place[1:])] = value
    return a


def refuses(f, args, status, message=None, **by_place):
    assert f(*changed(args, **by_place)) == status, (by_place, cb.lib().cascade_last_error())
    if message:
        assert message in cb.lib().cascade_last_error(), cb.lib().cascade_last_error()


def test_rope_rows(L):
    S = cb.Strides(0, 512, 128)
    args = [1, 4, 4, 128, 64, 0, P, S, P, P, 10, P, S, None]
    for place in ("6", "8", "9", "11"):
        refuses(L.cascade_rope_rows, args, 1, b"null", **{"_" + place: None})
    refuses(L.cascade_rope_rows, args, 3, _0=7)
    refuses(L.cascade_rope_rows, args, 3, b"head_dim 96", _3=96)
    for rot in (0, 8, 24, 144, -16):
        refuses(L.cascade_rope_rows, args, 3, b"rot_dim", _4=rot)
    refuses(L.cascade_rope_rows, args, 1, _1=0)
    refuses(L.cascade_rope_rows, args, 1, _2=0)
    refuses(L.cascade_rope_rows, args, 3, _2=65536)
    refuses(L.cascade_rope_rows, args, 1, _10=0)
    refuses(L.cascade_rope_rows, args, 1, b"aligned", _6=P + 8)
    refuses(L.cascade_rope_rows, args, 1, b"aligned", _7=cb.Strides(0, 508, 128))
    refuses(L.cascade_rope_rows, args, 1, b"aligned", _12=cb.Strides(0, 512, 127))


def test_scaled_table(L):
    args = [100, 64, 10000.0, 3, 8.0, 4096.0, 1.0, 4.0, 0.0, P, None]
    f, nan = L.cascade_rope_table_scaled, float("nan")
    for place, values in ((0, [0, -1]), (1, [0, 63]), (2, [1.0, nan, float("inf")]), (3, [-1, 5]), (4, [0.5, nan]), (5, [0.0, nan]),
                          (6, [0.0, 4.0, nan]), (7, [1.0, nan]), (8, [-1.0, nan]), (9, [None, P + 4])):
        for v in values:
            refuses(f, args, 1, **{f"_{place}": v})
    refuses(f, args, 1, _1=2, _3=2)  # a scaled base needs more than two columns
    with pytest.raises(cb.CascadeError, match="unknown kind"):
        cb.cascade_rope_table_scaled(10, 64, 10000.0, "other", device="cpu")


def test_append(L):
    S, G = cb.Strides(0, 512, 128), cb.Strides(16 * 512, 512, 128)
    #        0  1  2  3  4   5   6  7  8  9  10 11 12 13  14    15 16  17 18 19 20 21 22 23  24 25 26 27 28 29 30
    args = [1, 2, 4, 8, 4, 128, P, S, P, S, P, S, P, S, None, P, 64, 128, 0, P, G, P, G, 9, 16, P, 5, 5, P, P, None]
    f = L.cascade_paged_append
    for place in (10, 12, 19, 21, 25, 28, 29, 8):
        refuses(f, args, 1, b"null", **{f"_{place}": None})
    refuses(f, args, 3, _0=2)
    refuses(f, args, 3, _5=32)
    refuses(f, args, 3, b"rot_dim", _17=136)
    refuses(f, args, 3, b"page_size", _24=24)
    refuses(f, args, 3, b"page_size", _24=8)
    for place in (1, 2, 3, 4, 23, 27, 16):
        refuses(f, args, 1, **{f"_{place}": 0})
    refuses(f, args, 1, _26=4)  # rows of the table closer together than they are long
    refuses(f, args, 3, b"2^30", _24=1 << 28)
    refuses(f, args, 1, b"aligned", _20=cb.Strides(16 * 512 + 4, 512, 128))
    refuses(f, args, 1, b"aligned", _10=P + 2)
    refuses(f, args, 1, _28=P + 2)


def test_attention(L):
    S, G = cb.Strides(0, 512, 128), cb.Strides(16 * 512, 512, 128)
    #        0  1  2  3  4  5   6    7   8  9 10 11 12 13 14 15  16 17 18 19 20 21   22  23 24    25   26 27    28
    args = [1, 2, 4, 3, 8, 4, 128, 0.1, 1, P, S, P, G, P, G, 9, 16, P, 5, 5, P, P, None, P, S, None, P, 1 << 40, None]
    f = L.cascade_attn_paged
    for place in (9, 11, 13, 17, 20, 21, 23):
        refuses(f, args, 1, b"null", **{f"_{place}": None})
    for place in (1, 2, 3, 4, 5, 15, 19):
        refuses(f, args, 1, **{f"_{place}": 0})
    refuses(f, args, 3, b"multiple", _4=9)
    refuses(f, args, 3, _0=-1)
    refuses(f, args, 3, _6=256)
    refuses(f, args, 3, b"page_size", _16=40)
    for scale in (0.0, -1.0, float("nan"), float("inf")):
        refuses(f, args, 1, b"scale", _7=scale)
    refuses(f, args, 1, b"aligned", _9=P + 8)
    refuses(f, args, 1, b"aligned", _22=P + 2)
    refuses(f, args, 1, b"aligned", _25=P + 2)
    refuses(f, args, 1, b"aligned", _12=cb.Strides(16 * 512, 512, 132))
    refuses(f, args, 3, _1=65536)
    n = ctypes.c_size_t()
    sizes = [0, 1, 32, 32, 8, 2, 64, 16, 4096]
    assert L.cascade_attn_paged_workspace_bytes(*sizes, ctypes.byref(n)) == 0 and n.value > 0
    refuses(f, args, 4, b"workspace", _0=0, _1=1, _2=32, _3=32, _4=8, _5=2, _6=64, _18=4096, _19=4096, _27=n.value - 1)
    refuses(f, args, 4, b"workspace", _0=0, _1=1, _2=32, _3=32, _4=8, _5=2, _6=64, _18=4096, _19=4096, _26=None)
    refuses(f, args, 4, b"workspace", _0=0, _1=1, _2=32, _3=32, _4=8, _5=2, _6=64, _18=4096, _19=4096, _26=P + 16)
    for place in range(1, 9):
        bad = list(sizes)
        bad[place] = 0
        assert L.cascade_attn_paged_workspace_bytes(*bad, ctypes.byref(n)) in (1, 3)
    assert L.cascade_attn_paged_workspace_bytes(*sizes, None) == 1


def test_page_tables(L):
    fork = [4, 3, 9, 16, P, P, P, P, 2 * P, 2 * P, 3 * P, 4 * P, 5 * P, None]
    for place in range(4):
        refuses(L.cascade_pages_fork, fork, 1, **{f"_{place}": 0})
    for place in range(4, 13):
        refuses(L.cascade_pages_fork, fork, 1, b"null", **{f"_{place}": None})
    refuses(L.cascade_pages_fork, fork, 3, b"8192", _0=8193)
    refuses(L.cascade_pages_fork, fork, 3, _3=1 << 30)
    refuses(L.cascade_pages_fork, fork, 1, b"table", _8=P)
    refuses(L.cascade_pages_fork, fork, 1, b"lengths", _9=P)
    refuses(L.cascade_pages_fork, fork, 1, b"aligned", _11=P + 4)
    compact = [4, 3, 9, 16, P, P, 2 * P, 3 * P, 4 * P, 5 * P, None]
    for place in range(4):
        refuses(L.cascade_pages_compact, compact, 1, **{f"_{place}": 0})
    for place in range(4, 10):
        refuses(L.cascade_pages_compact, compact, 1, b"null", **{f"_{place}": None})
    refuses(L.cascade_pages_compact, compact, 1, b"table", _6=P)
    pools, strides = (ctypes.c_void_p * 2)(P, 2 * P), (ctypes.c_int64 * 2)(512, 512)
    copy = [2, pools, strides, 512, 9, P, 3, None]
    f = L.cascade_pages_copy
    for place in (1, 2, 5):
        refuses(f, copy, 1, b"null", **{f"_{place}": None})
    for place, value in ((0, 0), (3, 0), (3, 24), (4, 0), (6, -1)):
        refuses(f, copy, 1, **{f"_{place}": value})
    refuses(f, copy, 3, b"257", _0=257)
    refuses(f, copy, 1, _2=(ctypes.c_int64 * 2)(512, 496))
    refuses(f, copy, 1, _2=(ctypes.c_int64 * 2)(512, 520))
    refuses(f, copy, 1, _1=(ctypes.c_void_p * 2)(P, P + 8))
    assert f(*changed(copy, _6=0)) == 0  # nothing to copy
    assert L.cascade_paged_status(None) == 1


def test_the_binding_takes_tensors_of_the_current_device_only(L):
    x, pos, table = torch.zeros(2, 2, 64), torch.zeros(2, dtype=torch.int32), torch.zeros(4, 32, 2)
    with pytest.raises(ValueError, match="GPU"):
        cb.cascade_rope_rows(x, pos, table)
    pages, ids = torch.zeros(3, 16, 2, 64), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        cb.cascade_attn_paged(x, pages, pages, ids, pos, pos[:1], 1.0)
    with pytest.raises(ValueError, match="GPU"):
        cb.cascade_paged_append(x, x, pages, pages, ids, pos, pos[:1])
    for call in (lambda: cb.cascade_pages_fork(ids, pos[:1], pos[:1], pos[:1], 3, 16), lambda: cb.cascade_pages_compact(ids, pos[:1], 3, 16),
                 lambda: cb.cascade_pages_copy([pages], ids)):
        with pytest.raises(ValueError, match="GPU"):
            call()
    with pytest.raises(TypeError):
        cb.cascade_rope_rows(None, pos, table)


def test_more_rows_of_cache_than_32_bits_number_blocks_of(L):
    """Sixteen rows are a block, and the blocks of all sequences are counted in 32 bits."""
    S, G = cb.Strides(0, 512, 128), cb.Strides(16 * 512, 512, 128)
    args = [1, 32, 32, 1, 8, 4, 128, 0.1, 1, P, S, P, G, P, G, 9, 16, P, 1 << 26, 1 << 26, P, P, None, P, S, None, P, 1 << 40, None]
    refuses(L.cascade_attn_paged, args, 3, b"2^35")
    n = ctypes.c_size_t()
    assert L.cascade_attn_paged_workspace_bytes(1, 32, 32, 1, 8, 4, 128, 16, 1 << 26, ctypes.byref(n)) == 3
    assert L.cascade_attn_paged_workspace_bytes(1, 31, 32, 1, 8, 4, 128, 16, 1 << 26, ctypes.byref(n)) == 0


def test_tables_beyond_32_bits(L):
    fork = [4, 3, 9, 16, P, P, P, P, 2 * P, 2 * P, 3 * P, 4 * P, 5 * P, None]
    compact = [4, 3, 9, 16, P, P, 2 * P, 3 * P, 4 * P, 5 * P, None]
    for f, args in ((L.cascade_pages_fork, fork), (L.cascade_pages_compact, compact)):
        refuses(f, args, 3, b"pages", _2=(1 << 30) + 1)
        refuses(f, args, 3, b"entries", _0=8192, _1=1 << 18)
    pools, strides = (ctypes.c_void_p * 1)(P), (ctypes.c_int64 * 1)(512)
    refuses(L.cascade_pages_copy, [1, pools, strides, 512, 9, P, (1 << 30) + 1, None], 3, b"pairs")
