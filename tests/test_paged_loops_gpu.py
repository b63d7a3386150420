"""Loops on PagedCache as a server runs them: steps captured in a graph and replayed, models of many layers."""
import math

import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2507_05228_b200 import binding as cb
from paper_2507_05228_b200.paged import PagedCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,page", [(torch.bfloat16, 128, 16), (torch.bfloat16, 64, 48), (torch.float32, 64, 16)])
def test_a_captured_step_goes_on_from_replay_to_replay(dtype, d, page):
    """Fork, append and attention of a token for every sequence in one graph: lengths grow over page boundaries, sequences fork and end
    between replays, and eager steps and compactions come between them."""
    rng, g = np.random.default_rng(page + d), torch.Generator().manual_seed(d)
    seqs, layers, H, Hkv, most, scale = 5, 2, 8, 2, 200, 1 / math.sqrt(d)
    cache = PagedCache(layers, 90 if page == 16 else 40, page, Hkv, d, seqs, most, dtype)
    for t in cache.k + cache.v:
        t.fill_(math.nan)
    none = torch.zeros(0, Hkv, d, dtype=dtype)
    held, lens = [[(none, none)] * layers for _ in range(seqs)], [0] * seqs
    fixed = [{n: torch.zeros(seqs, h, d, dtype=dtype, device="cuda") for n, h in (("q", H), ("k", Hkv), ("v", Hkv))} for _ in range(layers)]
    source, add, row_start = pu.ints(np.arange(seqs)), pu.ints(np.ones(seqs)), pu.ints(np.arange(seqs + 1))
    results = [None] * layers

    def step():
        cache.step(source, add)
        for x in range(layers):
            cache.append(x, fixed[x]["k"], fixed[x]["v"], row_start)
            results[x] = cache.attend(x, fixed[x]["q"], row_start, scale, max_rows=1)

    def new_rows():
        for x in range(layers):
            for t in fixed[x].values():
                t.copy_(torch.randn(t.shape, generator=g).to(dtype))

    def follow(src, what):
        nonlocal held, lens
        held = [[tuple(torch.cat([held[s][x][j] if s >= 0 else none, fixed[x][n][i:i + 1].cpu()]) for j, n in enumerate("kv"))
                 for x in range(layers)] for i, s in enumerate(src)]
        lens = [(lens[s] if s >= 0 else 0) + 1 for s in src]
        assert cache.kv_len.tolist() == lens and not cache.report[:3].any().item(), what
        assert cache.refs.sum().item() == sum(-(-x // page) for x in lens), what
        for x in range(layers):
            b = pu.Batch.__new__(pu.Batch)
            b.rows, b.lens, b.starts, b.n, b.H, b.Hkv, b.d, b.dtype, b.scale = [1] * seqs, lens, np.arange(seqs + 1), seqs, H, Hkv, d, dtype, scale
            b.q64 = fixed[x]["q"].double().cpu()
            b.k_rows, b.v_rows = [s[x][0].double() for s in held], [s[x][1].double() for s in held]
            b.check(*results[x], what=(what, x))

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        new_rows()
        step()
    torch.cuda.synchronize()
    follow(range(seqs), "eager")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    captured = list(results)
    for turn in range(2 * page + 5):
        src = list(range(seqs))
        if turn % 7 == 3:
            src[turn % seqs] = -1
        if turn % 4 == 1:
            src = [int(s) for s in rng.integers(0, seqs, seqs)]
        source.copy_(pu.ints(src))
        new_rows()
        if turn % 9 == 8:
            step()  # outside the graph
            follow(src, (turn, "eager"))
        else:
            graph.replay()
            results[:] = captured
            follow(src, turn)
        if turn % 11 == 10:
            report = cache.compact()
            assert report[2].item() == 0 and cache.refs[:report[0].item()].all().item()
    assert cb.cascade_paged_status() == 0


def test_a_model_of_more_layers_than_a_copy_takes_pools():
    layers, page, Hkv, d = 130, 16, 1, 64
    cache = PagedCache(layers, 6, page, Hkv, d, 2, 64)
    cache.step(pu.ints([-1, -1]), pu.ints([20, 0]))
    first, second = cache.table[0, :2].tolist()
    for x in range(layers):
        cache.k[x].fill_(0)
        cache.v[x].fill_(0)
        cache.k[x][second], cache.v[x][second] = 1 + x, 1000 + x
    cache.step(pu.ints([0, 0]), pu.ints([0, 1]))
    assert cache.report[:3].tolist() == [0, 0, 0] and cache.table[0, :2].tolist() == [first, second]
    mine = cache.table[1, 1].item()
    assert cache.table[1, 0].item() == first and mine != second
    for x in range(layers):
        assert torch.equal(cache.k[x][mine], cache.k[x][second]) and torch.equal(cache.v[x][mine], cache.v[x][second]), x
    cache.step(pu.ints([-1, 1]), pu.ints([0, 0]))
    report = cache.compact()
    assert report[:3].tolist() == [2, 1, 0] and sorted(cache.table[1, :2].tolist()) == [0, 1]
    for x in range(layers):
        assert (cache.k[x][cache.table[1, 1].item()] == 1 + x).all()
