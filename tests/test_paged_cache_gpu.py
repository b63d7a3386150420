"""A serving loop on PagedCache: prompts in chunks, tokens, drafts, forks, ended sequences, compaction, all layers; every step's
attention against 64 bits over lists of the rows that the sequences should hold."""
import math

import numpy as np
import pytest
import torch

import paged_util as pu
from paper_2507_05228_b200 import binding as cb
from paper_2507_05228_b200.paged import PagedCache

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,page,interleaved,rot", [(torch.bfloat16, 128, 16, False, 128), (torch.bfloat16, 64, 48, True, 32),
                                                          (torch.float32, 64, 16, False, 64)])
def test_serving_loop(dtype, d, page, interleaved, rot):
    rng, g = np.random.default_rng(d + page), torch.Generator().manual_seed(page)
    seqs, layers, H, Hkv, most = 9, 2, 8, 2, 400
    cache = PagedCache(layers, 150 if page == 16 else 60, page, Hkv, d, seqs, most, dtype)
    for t in cache.k + cache.v:
        t.fill_(math.nan)
    table = cb.cascade_rope_table_scaled(most, rot, 10000.0, "linear", 2.0)
    held = [[(torch.zeros(0, Hkv, d, dtype=dtype),) * 2 for _ in range(layers)] for _ in range(seqs)]  # k, v of every layer
    lens = [0] * seqs
    for step in range(24):
        source, add = [], []
        for i in range(seqs):
            live = [j for j in range(seqs) if lens[j]]
            if rng.random() < 0.15:  # ended; perhaps a new prompt takes the place
                source.append(-1)
                add.append(int(rng.integers(0, 90)))
            elif live and rng.random() < 0.3:
                source.append(int(rng.choice(live)))
                add.append(int(rng.choice([0, 1, 1, 4])))
            else:
                source.append(i)
                add.append(int(rng.choice([0, 1, 1, 1, 5, 70])))
            have = lens[source[i]] if source[i] >= 0 else 0
            add[i] = min(add[i], most - have)
        copies = cache.step(pu.ints(source), pu.ints(add))
        if cache.report[:3].any().item():  # no room: a sequence ends instead
            assert cache.report[0].item() > 0 and (copies == -1).all() and cache.kv_len.tolist() == lens
            end = int(np.argmax(lens))
            cache.step(pu.ints([-1 if i == end else i for i in range(seqs)]), pu.ints([0] * seqs))
            lens[end] = 0
            held[end] = [(torch.zeros(0, Hkv, d, dtype=dtype),) * 2 for _ in range(layers)]
            continue
        held = [[held[s][x] if s >= 0 else (torch.zeros(0, Hkv, d, dtype=dtype),) * 2 for x in range(layers)] for s in source]
        lens = [(lens[s] if s >= 0 else 0) + a for s, a in zip(source, add)]
        assert cache.kv_len.tolist() == lens
        if step % 5 == 4:
            cache.compact()
        n, starts = sum(add), np.concatenate([[0], np.cumsum(add)])
        if n == 0:
            continue
        row_start = pu.ints(starts)
        positions = pu.ints(np.concatenate([np.arange(x - a, x) for x, a in zip(lens, add)]))
        for layer in range(layers):
            q, k, v = (torch.randn((n, h, d), generator=g).to(dtype).cuda() for h in (H, Hkv, Hkv))
            q_out = cache.append(layer, k, v, row_start, q=q, rope_table=table, interleaved=interleaved)
            k_turned = cb.cascade_rope_rows(k, positions, table, interleaved=interleaved).cpu()
            assert torch.equal(q_out, cb.cascade_rope_rows(q, positions, table, interleaved=interleaved))
            o, lse = cache.attend(layer, q_out, row_start, 1 / math.sqrt(d), max_rows=max(add))
            for i in range(seqs):
                r = slice(int(starts[i]), int(starts[i + 1]))
                held[i][layer] = (torch.cat([held[i][layer][0], k_turned[r]]), torch.cat([held[i][layer][1], v.cpu()[r]]))
            b = pu.Batch.__new__(pu.Batch)
            b.rows, b.lens, b.starts, b.n, b.H, b.Hkv, b.d, b.dtype, b.scale = add, lens, starts, n, H, Hkv, d, dtype, 1 / math.sqrt(d)
            b.q64 = q_out.double().cpu()
            b.k_rows, b.v_rows = [h[layer][0].double() for h in held], [h[layer][1].double() for h in held]
            b.check(o, lse, what=step)
        assert cache.refs.sum().item() == sum(-(-x // page) for x in lens)
    assert cb.cascade_paged_status() == 0
