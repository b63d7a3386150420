"""Plain 64-bit forms of the paged operators, and inputs for them."""
import math

import numpy as np
import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}  # a rounding, relative to the value


def ints(values, device="cuda"):
    return torch.tensor(np.asarray(values), dtype=torch.int32, device=device)


class Batch:
    """Ragged rows over paged caches.  rows[b] new rows and lens[b] cache rows of sequence b; everything that no length reaches is
    NaN, and the table's unused entries and the padded rows are garbage."""

    def __init__(self, rows, lens, H, Hkv, d, page, dtype=torch.bfloat16, seed=0, pad=3, head_major=False, lead=0, spare=3, scale_k=1.0,
                 strided=False, width=None):
        g = torch.Generator().manual_seed(seed)
        rng = np.random.default_rng(seed)
        self.rows, self.lens, self.H, self.Hkv, self.d, self.page, self.dtype = list(rows), list(lens), H, Hkv, d, page, dtype
        n = lead + sum(rows) + pad
        self.n = n
        self.starts = np.concatenate([[0], np.cumsum(rows)]) + lead
        counts = [-(-x // page) for x in lens]
        self.n_pages, width = sum(counts) + spare, width or max(counts + [1]) + 1
        table = rng.choice([-7, 2 ** 30, 10 ** 6], (len(rows), width)).astype(np.int32)
        ids = rng.permutation(self.n_pages)
        at = 0

        def normal(*shape):
            return torch.randn(shape, generator=g, dtype=torch.float32)

        shape = (self.n_pages, Hkv, page, d) if head_major else (self.n_pages, page, Hkv, d)
        pages = [torch.full(shape, math.nan, dtype=dtype) for _ in range(2)]
        if head_major:
            pages = [p.transpose(1, 2) for p in pages]
        self.k_rows, self.v_rows = [], []
        for b, (c, x) in enumerate(zip(counts, lens)):
            table[b, :c] = ids[at:at + c]
            at += c
            k, v = (normal(x, Hkv, d) * scale_k).to(dtype), normal(x, Hkv, d).to(dtype)
            self.k_rows.append(k.double())
            self.v_rows.append(v.double())
            for y0 in range(0, x, page):
                e = min(x, y0 + page) - y0
                pages[0][table[b, y0 // page], :e] = k[y0:y0 + e]
                pages[1][table[b, y0 // page], :e] = v[y0:y0 + e]
        q = normal(n, H, d).to(dtype)
        self.q64 = q.double()

        def up(t):  # (keeps the order of the dimensions in memory)
            return t.cuda()

        self.k_pages, self.v_pages = up(pages[0]), up(pages[1])
        if head_major:
            self.k_pages, self.v_pages = (p.transpose(1, 2).contiguous().cuda().transpose(1, 2) for p in pages)
        if strided:  # q inside packed q, k, v rows
            packed = torch.empty((n, H + 2 * Hkv, d), dtype=dtype, device="cuda")
            packed[:, :H] = q.cuda()
            self.q = packed[:, :H]
        else:
            self.q = q.cuda()
        self.table, self.row_start, self.kv_len = ints(table), ints(self.starts), ints(lens)
        self.scale = 1 / math.sqrt(d)

    def seen(self, b, causal, visible):
        n, x = self.rows[b], self.lens[b]
        if visible is not None:
            return np.clip(np.asarray(visible)[self.starts[b]:self.starts[b + 1]], 0, x)
        return np.clip(x - n + np.arange(n) + 1, 0, x) if causal else np.full(n, x)

    def reference(self, causal=True, visible=None):
        """(o, lse) and how far a result may be off: (of o per element, of lse per row).

        Logits: a sum of d products in fp32, on the tensor cores with truncated additions, is off by at most d 2^-23 of the sum of
        their absolute values A; the largest weight difference that makes is 2 d 2^-23 A relative, and as much again for the product
        with the scale and the exponential (2^-21).  Sums over n keys: n 2^-24.  bf16 weights: 2^-8 each.  All of these are
        relative to sum w |v|.  The output is rounded once."""
        o = torch.zeros(self.n, self.H, self.d, dtype=torch.float64)
        lse = torch.full((self.n, self.H), -math.inf, dtype=torch.float64)
        off_o, off_lse = torch.zeros_like(o), torch.zeros_like(lse)
        G = self.H // self.Hkv
        for b in range(len(self.rows)):
            seen = self.seen(b, causal, visible)
            r = slice(int(self.starts[b]), int(self.starts[b + 1]))
            hidden = torch.arange(self.lens[b]) >= torch.tensor(seen)[:, None]
            for h in range(self.H):
                if self.lens[b] == 0 or self.rows[b] == 0:
                    continue
                k, v, q = self.k_rows[b][:, h // G], self.v_rows[b][:, h // G], self.q64[r, h]
                a = (q @ k.T * self.scale).masked_fill(hidden, -math.inf)
                size = (q.abs() @ k.abs().T * self.scale).masked_fill(hidden, 0).amax(-1, keepdim=True)
                m = a.amax(-1, keepdim=True)
                w = torch.exp(a - torch.where(m == -math.inf, 0, m))
                total = w.sum(-1, keepdim=True)
                w = w / torch.where(total > 0, total, 1)
                o[r, h], lse[r, h] = w @ v, (m + total.log())[:, 0]
                small = 2 * self.d * 2.0 ** -23 * size + 2.0 ** -21 + self.lens[b] * 2.0 ** -24
                rounded = HALF[self.dtype] if self.dtype == torch.bfloat16 else 0
                off_o[r, h] = (w @ v.abs()) * (small + rounded) + HALF[self.dtype] * o[r, h].abs()
                off_lse[r, h] = small[:, 0] + 2.0 ** -23 * lse[r, h].abs().nan_to_num(posinf=0)
        return o, lse, off_o, off_lse

    def check(self, out, lse, causal=True, visible=None, o_before=None, what=""):
        o_ref, lse_ref, off_o, off_lse = self.reference(causal, visible)
        rows = torch.arange(self.n)
        mine = (rows >= int(self.starts[0])) & (rows < int(self.starts[-1]))
        got = out.double().cpu()
        assert torch.isfinite(got[mine]).all(), what
        over = ((got - o_ref).abs() - off_o)[mine]
        assert over.numel() == 0 or over.max() <= 0, (what, over.max().item(), (got - o_ref).abs()[mine].max().item())
        if o_before is not None:
            assert torch.equal(out.cpu()[~mine], o_before.cpu()[~mine]), what
        if lse is not None:
            l64 = lse.double().cpu()
            none = lse_ref == -math.inf
            assert torch.equal((l64 == -math.inf)[mine], none[mine]), what
            fine = mine[:, None] & ~none
            over = ((l64 - lse_ref).abs() - off_lse)[fine]
            assert over.numel() == 0 or over.max() <= 0, (what, over.max().item())


def turn(x, positions, table, interleaved):
    """x [rows, heads, d] in 64 bits turned by rows of the table [n, rot/2, 2]."""
    x, rot = x.double().clone(), 2 * table.shape[1]
    cs = table.double()[positions]
    by = torch.complex(cs[..., 0], cs[..., 1])[:, None]
    re, im = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    z = torch.complex(x[..., re], x[..., im]) * by
    x[..., re], x[..., im] = z.real, z.imag
    return x


def turn_bound(x, table, positions, dtype, rot, interleaved):
    """Two products and a sum in fp32 (three roundings of values no larger than |a c| + |b s|), then a rounding to the type."""
    t = turn(x.double().abs() * 1.0, positions, torch.stack([table[..., 0].abs(), -table[..., 1].abs()], -1), interleaved)
    u = turn(x.double().abs(), positions, table.abs(), interleaved)
    size = torch.maximum(t.abs(), u.abs())
    turned = torch.zeros(x.shape[-1], dtype=torch.bool)
    turned[:rot] = True
    return torch.where(turned, size * (3 * 2.0 ** -24 + HALF[dtype]) * (1 + 2.0 ** -8), 0.0)


def fork(table, kv_len, source, add, n_pages, page):
    """cascade_pages_fork with lists: (table, kv_len, refs, copies, report)."""
    n, width = table.shape
    old = [[int(p) for p in table[i][:-(-int(kv_len[i]) // page)]] if 0 <= kv_len[i] <= width * page else None for i in range(n)]

    def refused(lacking, long, bad):
        refs = [0] * n_pages
        for pages in old:
            for p in pages or []:
                if 0 <= p < n_pages:
                    refs[p] += 1
        return table.copy(), kv_len.copy(), np.array(refs), np.full((n, 2), -1), [lacking, long, bad, refs.count(0)]

    lists, had, bad, long = [], [], 0, 0
    for i in range(n):
        s, a, rows = int(source[i]), int(add[i]), 0
        if s < -1 or s >= n or a < 0:
            bad += 1
        elif s >= 0:
            if old[s] is None:
                bad += 1
            else:
                rows = int(kv_len[s])
        long += rows + max(a, 0) > width * page
        had.append(rows)
        lists.append(list(old[s]) if rows else [])
        bad += sum(not 0 <= p < n_pages for p in lists[-1])
    holders = {}
    for i, pages in enumerate(lists):
        for p in pages:
            holders.setdefault(p, []).append(i)
    writes = [had[i] % page != 0 and add[i] > 0 for i in range(n)]
    copied = []
    for i in range(n):
        if not writes[i] or not 0 <= lists[i][-1] < n_pages:
            copied.append(False)
            continue
        p = lists[i][-1]
        everyone = all(writes[j] and lists[j][-1] == p for j in holders[p])
        copied.append(len(holders[p]) > 1 and not (everyone and holders[p][0] == i))
    need = [-(-(had[i] + max(int(add[i]), 0)) // page) - len(lists[i]) + copied[i] for i in range(n)]
    free = [p for p in range(n_pages) if p not in holders]
    if bad or long or sum(need) > len(free):
        return refused(max(0, sum(need) - len(free)), long, bad)
    copies, at = np.full((n, 2), -1), 0
    for i in range(n):
        mine = free[at:at + need[i]]
        at += need[i]
        if copied[i]:
            copies[i] = lists[i][-1], mine[0]
            lists[i][-1] = mine.pop(0)
        lists[i] += mine
    out = np.full((n, width), -1)
    refs = np.zeros(n_pages, int)
    for i, pages in enumerate(lists):
        out[i, :len(pages)] = pages
        for p in pages:
            refs[p] += 1
    return out, np.array([had[i] + int(add[i]) for i in range(n)]), refs, copies, [0, 0, 0, len(free) - at]


def compact(table, kv_len, n_pages, page):
    n, width = table.shape
    held = sorted({int(p) for i in range(n) for p in table[i][:-(-int(kv_len[i]) // page)]})
    holes = [p for p in range(len(held)) if p not in set(held)]
    movers = [p for p in held if p >= len(held)]
    to = dict(zip(movers, holes))
    out, refs = np.full((n, width), -1), np.zeros(n_pages, int)
    for i in range(n):
        for c in range(-(-int(kv_len[i]) // page)):
            out[i, c] = to.get(int(table[i, c]), int(table[i, c]))
            refs[out[i, c]] += 1
    moves = np.full((n_pages // 2, 2), -1)
    for j, m in enumerate(movers):
        moves[j] = m, to[m]
    return out, refs, moves, [len(held), len(movers), 0, n_pages - len(held)]
