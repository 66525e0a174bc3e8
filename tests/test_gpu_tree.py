"""Trees of drafted tokens on the GPU: layout, accepted paths, rows moved between slots, attention of trees over pages, each against a plain implementation."""
import random

import pytest
import torch

pytestmark = pytest.mark.gpu

T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def binding():
    from paper_2602_16760_amd import binding as B
    return B


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def i64(values):
    return torch.tensor([v - (1 << 64) if v >> 63 else v for v in values], dtype=torch.int64, device="cuda")


def random_tree(rng, n):
    """Parents of n rows, some of which hang on nothing, on themselves or on a row behind them."""
    way = rng.randrange(4)
    parent = [rng.randint(-3, n)]  # (row 0's is not looked at)
    for j in range(1, n):
        x = rng.random()
        parent.append(rng.choice([-1, j, j + 1, 64, 2 ** 31 - 1, -2 ** 31]) if x < 0.06 else [j - 1, max(0, j - rng.randint(1, 5)), (j - 1) // 2, rng.randrange(j)][way])
    return parent[:n]


def paths(parent):
    """(depth, mask) of a block's rows by the published rules."""
    out = []
    for j, p in enumerate(parent):
        if j == 0:
            out.append((0, 1))
        elif j < 64 and 0 <= p < j and out[p][1]:
            out.append((out[p][0] + 1, out[p][1] | 1 << j))
        else:
            out.append((-1, 0))
    return out


# ---- la_tree_layout ----------------------------------------------------------------------------------------
@pytest.mark.parametrize("counts,front,pad", [([1], 0, 0), ([8], 0, 0), ([64], 0, 3), ([0, 5, 0, 64, 1, 33, 0], 0, 7), ([70, 3, 200], 0, 0), ([7] * 65, 2, 400), ([0], 0, 5),
                                              ([3 + r % 60 for r in range(700)], 0, 1)])
def test_layout(counts, front, pad):
    rng = random.Random(len(counts))
    first, parent, want = [front], [5] * front, [(-1, 0)] * front
    lens = [rng.randint(0, 100000) for _ in counts]
    for n, L in zip(counts, lens):
        tree = random_tree(rng, n)
        parent += tree
        want += [(L + d if m else -1, m) for d, m in paths(tree)]
        first.append(len(parent))
    parent += [0] * pad
    want += [(-1, 0)] * pad
    pos, vis = i32([77] * len(parent)), i64([77] * len(parent))
    binding().la_tree_layout(i32(parent), i32(first), i32(lens), pos, vis)
    assert pos.tolist() == [p for p, _ in want]
    assert vis.tolist() == i64([m for _, m in want]).tolist()


def test_layout_of_a_chain_is_the_causal_block_and_of_no_row_nothing():
    B = binding()
    pos, vis = i32([0] * 64), i64([0] * 64)
    B.la_tree_layout(i32([j - 1 for j in range(64)]), i32([0, 64]), i32([1000]), pos, vis)
    want_pos, want_vis = B.la_causal_layout(1000, 64)
    assert pos.tolist() == want_pos.tolist() and vis.tolist() == i64([int(v) for v in want_vis]).tolist()
    B.la_tree_layout(i32([]), i32([0, 0, 0]), i32([4, 5]), i32([]), i64([]))


# ---- la_tree_accept ----------------------------------------------------------------------------------------
def accept_by_hand(parent, tok, ids, slot, L, limit, max_path, f):
    """One request's results; f: its first row."""
    path, emitted, n = [], [], min(64, len(parent))
    while n and limit > 0:
        path.append(0 if not path else nxt)
        chosen = ids[path[-1]]
        if chosen < 0:
            break
        emitted.append(chosen)
        fits = [j for j in range(path[-1] + 1, n) if parent[j] == path[-1] and tok[j] == chosen]
        if len(emitted) == min(limit, max_path) or not fits:
            break
        nxt = fits[0]
    pad = lambda v: v + [-1] * (max_path - len(v))
    moves = [(slot[j], slot[k]) if j != k and slot[j] >= 0 and slot[k] >= 0 else (-1, -1) for k, j in enumerate(path)]
    return len(emitted), L + len(path), f + path[-1] if path else -1, pad(emitted), pad([a for a, _ in moves]), pad([b for _, b in moves])


@pytest.mark.parametrize("counts,max_path,limits", [([1], 1, None), ([8], 4, None), ([64, 0, 33, 1], 64, None), ([70, 12, 90], 8, None), ([12] * 40, 6, [0, 1, 2, 3, -5, 100]),
                                                    ([1 + r % 64 for r in range(600)], 16, [100, 100, 2, 0])])
@pytest.mark.parametrize("seed", [0, 1])
def test_accept(counts, max_path, limits, seed):
    rng = random.Random(seed)
    parent, tok, ids, slot, first, want = [], [], [], [], [0], []
    lens = [rng.randint(0, 1000) for _ in counts]
    limit = None if limits is None else [limits[r % len(limits)] for r in range(len(counts))]
    for r, n in enumerate(counts):
        tree = random_tree(rng, n)
        t = [rng.choice([-1, 0, 1, 2, 5]) for _ in range(n)]  # (few tokens: siblings with the same one; negative ones are never chosen)
        c = [rng.choice([0, 1, 2, 5, 5, 7]) for _ in range(n)]
        for j in range(n - 1, 0, -1):
            if rng.random() < 0.7 and 0 <= tree[j] < j:
                c[tree[j]] = t[j]
        c = [rng.choice([-1, -7]) if rng.random() < 0.05 else x for x in c]
        s = [rng.randrange(10000) if rng.random() < 0.95 else -1 for _ in range(n)]
        want.append(accept_by_hand(tree, t, c, s, lens[r], 1000 if limit is None else limit[r], max_path, first[-1]))
        parent, tok, ids, slot = parent + tree, tok + t, ids + c, slot + s
        first.append(len(parent))
    R = len(counts)
    got = [i32([77] * R) for _ in range(3)] + [torch.full((R, max_path), 77, dtype=torch.int32, device="cuda") for _ in range(3)]
    binding().la_tree_accept(i32(parent), i32(tok), i32(ids), i32(slot), i32(first), i32(lens), *got, limit=None if limit is None else i32(limit))
    for name, g, w in zip(("n_new", "new_len", "last", "out", "from", "to"), got, zip(*want)):
        assert g.tolist() == list(w), name


def test_accept_of_no_rows():
    got = [i32([77] * 2) for _ in range(3)] + [torch.full((2, 3), 77, dtype=torch.int32, device="cuda") for _ in range(3)]
    none = i32([])
    binding().la_tree_accept(none, none, none, none, i32([0, 0, 0]), i32([9, 0]), *got)
    assert [g.tolist() for g in got] == [[0, 0], [9, 0], [-1, -1]] + [[[-1] * 3] * 2] * 3


# ---- la_paged_copy -----------------------------------------------------------------------------------------
def copy_by_hand(pages, page, begin, end, frm, to, run):
    """Run by run: all sources, then all destinations in order."""
    out = pages.clone()
    slots = pages.shape[1] * page
    for i in range(0, len(frm), run):
        moves = [(a, b) for a, b in zip(frm[i:i + run], to[i:i + run]) if 0 <= a < slots and 0 <= b < slots]
        rows = [out[begin:end, a // page, :, a % page].clone() for a, _ in moves]
        for (_, b), row in zip(moves, rows):
            out[begin:end, b // page, :, b % page] = row
    return out


@pytest.mark.parametrize("dtype,layers,Hkv,dh,page", [("bf16", 3, 8, 128, 16), ("f16", 2, 2, 64, 5), ("f32", 2, 3, 80, 16), ("bf16", 1, 1, 8, 1), ("f32", 40, 1, 256, 24)])
@pytest.mark.parametrize("run", [1, 2, 7, 8, 9, 64])
def test_copy(dtype, layers, Hkv, dh, page, run):
    """Runs whose rows are each other's destinations (paths, swaps, circles), the same destination twice in one, pairs that are none, a last run that is shorter."""
    rng, B = random.Random(run * dh), binding()
    runs = 5
    n_pages = runs * run * 2 // page + 4
    g = torch.Generator().manual_seed(dh)
    k, v = (torch.randn((layers, n_pages, Hkv, page, dh), generator=g).to(T[dtype]) for _ in range(2))
    slots, frm, to = rng.sample(range(n_pages * page), runs * run * 2), [], []
    for r in range(runs):
        mine = slots[2 * r * run:2 * (r + 1) * run]
        a, b = [rng.choice(mine) for _ in range(run)], [rng.choice(mine) for _ in range(run)]  # (anything, twice the same among it)
        if r == 1:
            a, b = mine[1:run + 1], mine[:run]  # a path that moves up by one
        if r == 2:
            a, b = mine[:run], mine[1:run] + mine[:1]  # a circle
        frm, to = frm + a, to + b
    frm[-1], to[0] = -1, n_pages * page
    frm, to = frm[:len(frm) - run // 2], to[:len(to) - run // 2]
    begin, end = (0, layers) if run % 2 else (layers // 2, layers)
    pages = B.la_pages(k.cuda(), v.cuda())
    B.la_paged_copy(pages, i32(frm), i32(to), run=run, layers=(begin, end))
    for got, was in ((pages.k, k), (pages.v, v)):
        assert torch.equal(got.cpu(), copy_by_hand(was, page, begin, end, frm, to, run))


def test_copy_of_whole_requests_and_rows_as_runs():
    """A prompt's positions into pages of another request; two dimensions are runs."""
    B, page = binding(), 16
    k, v = (torch.randn((4, 200, 2, page, 64), generator=torch.Generator().manual_seed(s)).to(torch.bfloat16) for s in (1, 2))
    pages = B.la_pages(k.cuda(), v.cuda())
    order = torch.randperm(200 * page, generator=torch.Generator().manual_seed(3))
    frm, to = order[:1500].to(torch.int32), order[1500:3000].to(torch.int32)
    B.la_paged_copy(pages, frm.cuda(), to.cuda())
    want = [copy_by_hand(t, page, 0, 4, frm.tolist(), to.tolist(), 1) for t in (k, v)]
    assert torch.equal(pages.k.cpu(), want[0]) and torch.equal(pages.v.cpu(), want[1])
    swap = torch.tensor([[3, 4], [100, 101], [-1, -1]], dtype=torch.int32)
    B.la_paged_copy(pages, swap.cuda(), swap.flip(1).contiguous().cuda())
    want = [copy_by_hand(t, page, 0, 4, swap.flatten().tolist(), swap.flip(1).flatten().tolist(), 2) for t in want]
    assert torch.equal(pages.k.cpu(), want[0]) and torch.equal(pages.v.cpu(), want[1])


def test_copy_behind_32_bits():
    """Slots whose offsets pass 2^32 bytes in a layer, and a layer that begins behind them."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    B = binding()
    n_pages = (5 << 30) // (16 * 8 * 128 * 2)
    k = torch.empty((2, n_pages, 8, 16, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    slots = [0, 5, n_pages * 8 + 3, n_pages * 16 - 1]
    rows = torch.randn((2, 2, 4, 8, 128), device="cuda").to(torch.bfloat16)
    for t, x in ((k, rows[0]), (v, rows[1])):
        for i, s in enumerate(slots):
            t[:, s // 16, :, s % 16] = x[:, i]
    B.la_paged_copy(B.la_pages(k, v), i32(slots), i32(slots[::-1]), run=4)
    for t, x in ((k, rows[0]), (v, rows[1])):
        for i, s in enumerate(slots):
            assert torch.equal(t[:, s // 16, :, s % 16], x[:, 3 - i])


def test_copy_as_many_pairs_as_there_are_numbers():
    """2^31 - 1 pairs, all but a few of none."""
    if torch.cuda.mem_get_info()[0] < 40 << 30:
        pytest.skip("not enough memory")
    B = binding()
    n = 2 ** 31 - 1
    k, v = (torch.arange(2 * 16 * 8, dtype=torch.float32, device="cuda").reshape(1, 2, 1, 16, 8).to(torch.bfloat16) + t for t in range(2))
    frm, to = (torch.full((n,), -1, dtype=torch.int32, device="cuda") for _ in range(2))
    for at, (f, t) in ((0, (3, 20)), (64, (5, 21)), (n // 2, (7, 22)), (n - 1, (9, 23))):
        frm[at], to[at] = f, t
    want = []
    for x in (k, v):
        y = x.clone()
        for f, t in ((3, 20), (5, 21), (7, 22), (9, 23)):
            y[0, t // 16, 0, t % 16] = x[0, 0, 0, f]
        want.append(y)
    B.la_paged_copy(B.la_pages(k, v), frm, to, run=64)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


# ---- la_paged_tree_attend ------------------------------------------------------------------------------------
class Case:
    """Pages in any order, NaN wherever no request has a position; a request's keys are its committed positions and its block's rows."""

    def __init__(self, dtype, Hq, Hkv, dh, page, lens, counts, seed=0, spread=1.0, blocks=None, layers=1, back=0, masks=None):
        g, rng = torch.Generator().manual_seed(seed), random.Random(seed)
        self.dtype, self.Hq, self.Hkv, self.dh, self.page, self.lens, self.counts, self.g = T[dtype], Hq, Hkv, dh, page, lens, counts, g
        total = [max(0, n) + c for n, c in zip(lens, counts)]
        used = [(n + page - 1) // page for n in total]
        n_pages = sum(used) + 2
        order = torch.randperm(n_pages, generator=g).tolist()
        blocks = blocks or max(1, max(used))
        self.table = torch.full((len(lens), blocks), -1, dtype=torch.int32)
        self.k, self.v = (torch.full((layers, n_pages, Hkv, page, dh), float("nan"), dtype=self.dtype) for _ in range(2))
        self.layer, self.keys, self.first, self.vis, at = layers - 1, [], [0], [], 0
        for r, n in enumerate(total):
            mine = order[at:at + used[r]]
            at += used[r]
            self.table[r, :used[r]] = torch.tensor(mine, dtype=torch.int32)
            k, v = ((torch.randn((n, Hkv, dh), generator=g)).to(self.dtype) for _ in range(2))
            self.keys.append((k, v))
            for b, p in enumerate(mine):
                part = slice(b * page, min(n, (b + 1) * page))
                m = part.stop - part.start
                self.k[layers - 1, p, :, :m] = k[part].transpose(0, 1)
                self.v[layers - 1, p, :, :m] = v[part].transpose(0, 1)
            self.vis += [m for _, m in paths(random_tree(rng, counts[r]))] if masks is None else masks[r]
            self.first.append(len(self.vis))
        self.vis += [1] * back  # (rows of no request)
        self.q = (torch.randn((len(self.vis), Hq, dh), generator=g) * spread).to(self.dtype)

    def place(self, r, t):
        return (self.layer, int(self.table[r, t // self.page]), slice(None), t % self.page)

    def run(self, max_rows=64, scale=None, lens=None):
        B = binding()
        out = torch.full(self.q.shape, 77.0, dtype=self.dtype, device="cuda")
        B.la_paged_tree_attend(B.la_pages(self.k.cuda(), self.v.cuda()), self.layer, self.q.cuda(), self.table.cuda(), i32(self.first), i32(self.lens if lens is None else lens),
                               i64(self.vis), max_rows, out, scale=scale)
        torch.cuda.synchronize()
        return out.cpu()

    def check(self, out, scale=None, max_rows=64, skip=lambda r, t: False, rows=None, but_nan=False):
        """Against float64, as la_paged_attend's rows are: a probability is rounded to the type (half a step of it), as is the output; scores are sums of dh float products, their error shifts a
        probability by as much relatively; the exponential and the sums over n keys add 2^-23 a term."""
        scale = self.dh ** -0.5 if scale is None else scale
        half, g = torch.finfo(self.dtype).eps / 2, self.Hq // self.Hkv
        for r, L in enumerate(self.lens):
            k, v = (t.double().repeat_interleave(g, 1) for t in self.keys[r])
            for i in range(self.first[r], self.first[r + 1]):
                if rows is not None and i not in rows:
                    continue
                n_rows, j0 = min(max_rows, self.counts[r], 64), i - self.first[r]
                see = [t for t in range(L)] + [L + j for j in range(n_rows) if self.vis[i] >> j & 1]
                see = [t for t in see if not skip(r, t)] if self.vis[i] and L >= 0 and j0 < n_rows else []
                if not see:
                    assert (out[i] == 0).all(), f"row {i} sees nothing"
                    continue
                ks, vs = k[see], v[see]
                s = torch.einsum("hd,nhd->hn", self.q[i].double(), ks) * scale
                size = torch.einsum("hd,nhd->hn", self.q[i].double().abs(), ks.abs()).amax(1) * abs(scale)
                w = torch.softmax(s, 1)
                want, mass = torch.einsum("hn,nhd->hd", w, vs), torch.einsum("hn,nhd->hd", w, vs.abs())
                shift = ((self.dh + 8) * 2.0 ** -24 * size)[:, None]
                tol = (half if self.dtype != torch.float32 else 0.0) * mass + half * want.abs() + 2 * shift * mass + (len(see) + 16) * 2.0 ** -23 * mass + 1e-30
                err = (out[i].double() - want).abs()
                assert ((err <= tol) | (torch.isnan(err) if but_nan else torch.zeros_like(err, dtype=torch.bool))).all(), f"row {i} (request {r}, {len(see)} keys): {float((err / tol).max()):.2f} of the bound"
        assert (out[self.first[-1]:] == 0).all()


SHAPES = [("bf16", 32, 8, 128, 16), ("f16", 8, 2, 128, 16), ("bf16", 6, 2, 64, 32), ("f32", 4, 2, 64, 24), ("bf16", 24, 2, 96, 16), ("f16", 16, 1, 256, 16), ("bf16", 32, 1, 128, 8),
          ("bf16", 20, 1, 64, 5), ("f16", 3, 3, 8, 1), ("f32", 6, 3, 80, 16), ("f32", 5, 1, 256, 3), ("bf16", 2, 2, 200, 48), ("f16", 17, 1, 128, 64), ("bf16", 8, 1, 256, 33),
          ("f16", 9, 1, 64, 16), ("bf16", 5, 5, 128, 16), ("f32", 8, 1, 128, 16)]


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page", SHAPES)
def test_attend_short_and_long_requests(dtype, Hq, Hkv, dh, page):
    """No committed position, ends inside a page, a tile and a block, blocks of no row to 64, rows of no request behind them."""
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 100, 127, 128, 129, 700, 5]
    counts = [3, 1, 16, 17, 0, 4, 33, 64, 1, 9, 2, 31, 32, 12, 0]
    c = Case(dtype, Hq, Hkv, dh, page, lens, counts, back=3)
    out = c.run()
    c.check(out)
    assert torch.equal(out, c.run())


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page,lens,counts", [
    ("bf16", 32, 8, 128, 16, [5000, 1, 900, 4096], [16, 16, 5, 1]), ("bf16", 8, 8, 64, 64, [20000], [64]), ("f32", 4, 2, 64, 24, [3001, 40, 3000], [10, 64, 1]),
    ("f16", 12, 1, 256, 16, [9000, 77], [7, 40]), ("bf16", 16, 2, 112, 20, [2500, 2501, 600], [8, 1, 63]), ("f16", 40, 1, 128, 16, [3000, 800], [64, 3]), ("f16", 32, 8, 128, 32, [6000, 2047], [64, 50])])
def test_attend_requests_cut_into_items(dtype, Hq, Hkv, dh, page, lens, counts):
    """Requests that several workgroups share and a second launch joins, beside ones that are not cut."""
    c = Case(dtype, Hq, Hkv, dh, page, lens, counts, seed=3, spread=2.0)
    out = c.run()
    c.check(out)
    assert torch.equal(out, c.run())


@pytest.mark.parametrize("rows,heads", [(1, 1), (1, 4), (2, 8), (5, 3), (8, 4), (16, 1), (17, 1), (16, 4), (33, 2), (64, 1), (64, 4), (64, 8), (9, 16), (64, 16)])
def test_attend_columns(rows, heads):
    """Every number of query heads and rows that share a key, short and cut."""
    for ctx in (90, 1500):
        c = Case("bf16", heads, 1, 64, 16, [ctx, 3], [rows, max(1, rows // 2)], seed=rows)
        c.check(c.run(max_rows=rows), max_rows=rows)


@pytest.mark.parametrize("R", [64, 65, 130, 300])
@pytest.mark.parametrize("ctx", [300, 2000])
def test_attend_many_requests(R, ctx):
    """More requests than a wave's lanes look up at once, with and without items."""
    lens, counts = [(37 * r) % ctx for r in range(R)], [(5 * r) % 4 for r in range(R)]
    c = Case("bf16", 4, 2, 64, 16, lens, counts, seed=R)
    c.check(c.run(max_rows=4), max_rows=4)


@pytest.mark.parametrize("dtype,Hkv,dh,page,rows,ctx", [("bf16", 1, 64, 16, 24, 300), ("f16", 2, 128, 16, 20, 1500), ("bf16", 2, 128, 24, 20, 1500), ("f16", 1, 256, 16, 33, 1200), ("f32", 2, 64, 16, 9, 1200)])
def test_attend_many_requests_of_many_rows(dtype, Hkv, dh, page, rows, ctx):
    """More than 64 requests whose rows and heads are many; some have none, one is much longer than the others."""
    R = 70
    lens, counts = [(37 * r) % 90 for r in range(R)], [(7 * r) % rows for r in range(R)]
    lens[5], counts[5], counts[11] = ctx, rows, rows
    c = Case(dtype, 4 * Hkv, Hkv, dh, page, lens, counts, seed=R)
    out = c.run(max_rows=rows)
    c.check(out, max_rows=rows, rows=[i for i in range(len(c.vis)) if i % 5 == 0 or c.first[5] <= i < c.first[6]])
    assert torch.equal(out, c.run(max_rows=rows))


@pytest.mark.parametrize("rows,ctx", [(3, 100), (3, 2000), (30, 100), (30, 2000)])
def test_attend_rows_in_front_of_the_first_request_and_behind_the_last(rows, ctx):
    """Rows of no request on both sides are zeros, at one launch and at two."""
    B = binding()
    c = Case("bf16", 8, 2, 128, 16, [ctx, 7], [rows, 2])
    q = torch.cat((c.q[:4], c.q, c.q[:3]))[:, :, :].contiguous()
    out = torch.full(q.shape, 77.0, dtype=c.dtype, device="cuda")
    B.la_paged_tree_attend(B.la_pages(c.k.cuda(), c.v.cuda()), 0, q.cuda(), c.table.cuda(), i32([f + 4 for f in c.first]), i32(c.lens), i64([1] * 4 + c.vis + [1] * 3), rows, out)
    n = len(c.vis)
    assert (out[:4] == 0).all() and (out[4 + n:] == 0).all()
    c.check(out[4:4 + n].cpu(), max_rows=rows)


@pytest.mark.parametrize("rows,ctx,page", [(4, 60, 16), (4, 1500, 16), (40, 60, 16), (40, 1500, 16), (6, 100, 12)])
def test_attend_queries_that_are_no_numbers(rows, ctx, page):
    """A NaN or an infinity in a row's query head reaches that head's output alone; a row that sees nothing has zeros whatever its query holds."""
    c = Case("bf16", 8, 2, 64, page, [ctx], [rows], masks=[[(2 << j) - 1 for j in range(rows - 1)] + [0]])
    c.q[0, 3, 5], c.q[1, 6, 0], c.q[rows - 1] = float("nan"), float("inf"), float("nan")
    out = c.run(max_rows=rows)
    assert torch.isnan(out[0, 3]).all() and (out[rows - 1] == 0).all()
    assert torch.isfinite(out[0, [0, 1, 2, 4, 5, 6, 7]]).all() and torch.isfinite(out[1, [0, 1, 2, 3, 4, 5, 7]]).all()
    c.check(out, max_rows=rows, rows=range(2, rows))


def test_attend_masks_of_any_kind():
    """Rows that do not see themselves, see later rows, see nothing but the committed positions of their own block, bits behind the block's rows."""
    full = (1 << 64) - 1
    masks = [[full, 0, 1 << 63, 0b1010, full << 20 & full, 0b100], [0, 0, 0], [1, 0, full]]
    c = Case("bf16", 8, 2, 128, 16, [50, 20, 0], [6, 3, 3], masks=masks)
    c.check(c.run())
    c.check(c.run(max_rows=6), max_rows=6)


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page,lens,counts", [
    ("bf16", 8, 2, 64, 16, [6000], [5]), ("f16", 8, 2, 128, 8, [700], [9]), ("f32", 4, 2, 80, 24, [2300], [4]), ("bf16", 16, 1, 256, 16, [4100], [3]), ("f16", 8, 1, 96, 16, [3000, 260], [12, 7]),
    ("bf16", 4, 1, 200, 16, [1300], [2]), ("bf16", 2, 2, 64, 16, [130], [1])])
def test_attend_few_requests_of_a_long_table(dtype, Hq, Hkv, dh, page, lens, counts):
    """Many items a request, whose records several waves share: numbers of them that the waves do not divide, fewer than waves; NaN and infinities in queries, scores of -inf and NaN."""
    blocks = 8192 // page
    c = Case(dtype, Hq, Hkv, dh, page, lens, counts, blocks=blocks)
    out = c.run()
    c.check(out)
    assert torch.equal(out, c.run())
    nan, inf, g = float("nan"), float("inf"), Hq // Hkv
    c.q[0, 0, 3], c.q[len(c.vis) - 1, 1 % Hq, 0] = nan, inf
    got = c.run()
    others = [h for h in range(1, Hq) if len(c.vis) > 1 or h != 1 % Hq]  # (of one row both are in it)
    assert torch.isnan(got[0, 0]).all() and torch.equal(got[0, others], out[0, others])
    keep = [i for i in range(1, len(c.vis) - 1)]
    assert torch.equal(got[keep], out[keep])
    c = Case(dtype, Hq, Hkv, dh, page, lens, counts, blocks=blocks)
    c.q[:] = c.q.abs() + 0.5
    for t in range(lens[0] + counts[0]):
        c.k[c.place(0, t)][0] = -inf  # (of one kv head, nothing but scores of -inf; of the others as before)
    c.v[c.place(0, lens[0] - 1)][Hkv - 1, 2] = inf
    got = c.run()
    sees = [i for i in range(counts[0]) if c.vis[i]]
    assert (got[:counts[0], :g].masked_fill(torch.isnan(got[:counts[0], :g]), 0.0) == 0).all()  # (weights of nothing: zeros, or NaN where V is infinite)
    if Hkv > 1:
        assert (got[sees, (Hkv - 1) * g:, 2] == inf).all() and torch.isfinite(got[sees, (Hkv - 1) * g:, 3:]).all() and (got[:counts[0], :g] == 0).all()


@pytest.mark.parametrize("max_rows", [1, 4, 15, 16, 17])
def test_attend_rows_behind_max_rows_see_nothing(max_rows):
    c = Case("bf16", 8, 2, 64, 16, [100, 30, 2000], [17, 5, 16])
    c.check(c.run(max_rows=max_rows), max_rows=max_rows)


def test_attend_lengths_that_are_none():
    """A negative length; a length behind the table's end."""
    c = Case("bf16", 4, 2, 64, 16, [48, 30], [5, 5])
    out = c.run(lens=[-1, 30])
    assert (out[:5] == 0).all()
    c.check(out, rows=range(5, 10))
    c = Case("bf16", 4, 2, 64, 16, [64, 64], [1, 2], blocks=5, masks=[[1], [3, 3]])
    out = c.run(lens=[2 ** 31 - 1, 64])  # (80 positions are the table's, 65 of them are the request's; those behind have no page's data)
    c.table[0, 4] = -1
    out = c.run(lens=[2 ** 31 - 1, 64])
    c.check(out, skip=lambda r, t: r == 0 and t >= 64)


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 12), ("f32", 12), ("f16", 64)])
def test_attend_pages_that_are_none(dtype, page):
    c = Case(dtype, 4, 2, 64, page, [200, 200, 10], [9, 3, 2])
    c.table[0, 1], c.table[1, :], c.table[2, 0] = -5, 1 << 20, -1
    out = c.run()
    c.check(out, skip=lambda r, t: (r == 0 and t // page == 1) or r == 1 or (r == 2 and t // page == 0))


@pytest.mark.parametrize("dtype,Hq,Hkv,dh", [("bf16", 8, 2, 128), ("f16", 12, 2, 96), ("bf16", 16, 4, 64), ("f16", 6, 1, 256)])
@pytest.mark.parametrize("page", [8, 16, 24, 40])
@pytest.mark.parametrize("cap", [0, 30000, 300000])
def test_attend_pages_of_eights_and_long_tables(dtype, Hq, Hkv, dh, page, cap):
    """Blocks of many columns whose stages of keys begin, end and change pages at any eight positions; the table's length decides how many columns share K and V, and how requests are cut.  A page
    of each long request is none."""
    lens, counts = [0, 1500, 333, 700, 8], [64, 60, 17, 33, 5]
    c = Case(dtype, Hq, Hkv, dh, page, lens, counts, seed=page + cap, blocks=cap // page or None)
    c.table[1, 3], c.table[3, 0] = -1, 1 << 30
    out = c.run()
    c.check(out, skip=lambda r, t: (r == 1 and t // page == 3) or (r == 3 and t < page))
    assert torch.equal(out, c.run())


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 8.0])
def test_attend_other_scales(dtype, scale):
    c = Case(dtype, 4, 1, 64, 16, [200, 33], [6, 20], seed=9)
    c.check(c.run(scale=scale), scale=scale)


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page,ctx", [("f32", 2, 1, 64, 16, 40), ("bf16", 2, 1, 64, 16, 40), ("bf16", 32, 2, 128, 16, 1500), ("f16", 8, 1, 256, 24, 100), ("f16", 8, 2, 96, 16, 900), ("f16", 8, 2, 64, 16, 1100),
                                                        ("bf16", 4, 1, 256, 32, 1000), ("f16", 4, 1, 128, 16, 50)])
def test_attend_values_that_other_rows_do_not_see(dtype, Hq, Hkv, dh, page, ctx):
    """K and V of infinities and NaN in a drafted row reach the rows that see it, in their own channels, and no other row."""
    values_that_other_rows_do_not_see(dtype, Hq, Hkv, dh, page, ctx)


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page,ctx", [("bf16", 8, 2, 128, 16, 1500), ("f16", 8, 2, 128, 8, 100), ("f16", 16, 2, 96, 24, 700), ("bf16", 4, 1, 64, 40, 900), ("f16", 8, 1, 256, 8, 300)])
def test_attend_values_that_other_rows_do_not_see_in_a_long_table(dtype, Hq, Hkv, dh, page, ctx):
    values_that_other_rows_do_not_see(dtype, Hq, Hkv, dh, page, ctx, blocks=(1 << 18) // page)


def values_that_other_rows_do_not_see(dtype, Hq, Hkv, dh, page, ctx, blocks=None):
    n = 40
    parent = [0, 0, 1, 0, 3, 0, 5, 6] + [0] * (n - 8)  # rows 2, 4 and 7 end three branches
    masks = [m for _, m in paths(parent)]
    c = Case(dtype, Hq, Hkv, dh, page, [ctx, 20], [n, 4], blocks=blocks, masks=[masks, [1, 3, 5, 7]])
    inf, nan = float("inf"), float("nan")
    c.v[c.place(0, ctx + 2)][:, 5] = inf      # seen by row 2 alone
    c.v[c.place(0, ctx + 3)][:, 7] = nan      # by rows 3 and 4
    c.v[c.place(0, ctx + 4)][:, 9] = -inf     # by row 4
    c.k[c.place(0, ctx + 7)][:, 1] = nan      # by row 7
    c.k[c.place(0, ctx + 20)] = inf           # by row 20
    c.v[c.place(0, ctx + 20)] = nan
    c.v[c.place(0, ctx + 33)][:, 0] = inf     # (another tile of keys)
    out = c.run()
    finite = [i for i in range(n + 4) if i not in (2, 3, 4, 7, 20, 33)]
    assert torch.isfinite(out[finite]).all()
    c.check(out, rows=finite)
    assert (out[2, :, 5] == inf).all() and torch.isfinite(out[2, :, 6:]).all() and torch.isfinite(out[2, :, :5]).all()
    assert torch.isnan(out[3, :, 7]).all() and torch.isfinite(out[3, :, 8:]).all()
    assert torch.isnan(out[4, :, 7]).all() and (out[4, :, 9] == -inf).all() and torch.isfinite(out[4, :, 10:]).all() and torch.isfinite(out[4, :, 8]).all()
    assert torch.isnan(out[7]).all() and torch.isnan(out[20]).all()
    assert (out[33, :, 0] == inf).all() and torch.isfinite(out[33, :, 1:]).all()
    # the other channels of rows that see them: as if those numbers were not there (a row's channels have nothing to do with each other)
    for r, t, ch in ((0, ctx + 2, 5), (0, ctx + 3, 7), (0, ctx + 4, 9), (0, ctx + 33, 0)):
        c.keys[r][1][t][:, ch] = 0.0
    got = out.clone()
    for row, chans in ((2, [5]), (3, [7]), (4, [7, 9]), (33, [0])):
        for ch in chans:
            got[row, :, ch] = float("nan")
    c.check(got, rows=(2, 3, 4, 33), but_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attend_committed_values_that_are_none(dtype):
    """An infinite V of a committed position reaches every row that has a mask, scores of -inf alone give zeros, and a request's NaN stays in it."""
    c = Case(dtype, 2, 1, 64, 16, [40, 20, 33, 8], [3, 2, 4, 5], masks=[[1, 3, 0], [1, 2], [1, 3, 5, 0], [1, 3, 7, 15, 31]])
    c.v[c.place(0, 39)][:, 5] = float("inf")
    c.k[c.layer, c.table[1, :2].long()] = float("-inf")
    c.q[3:5] = c.q[3:5].abs() + 0.5
    c.k[c.place(2, 30)][:, 3] = float("nan")
    out = c.run()
    assert torch.isinf(out[:2, :, 5]).all() and torch.isfinite(out[:2, :, 6:]).all() and (out[2] == 0).all()
    assert (out[3:5] == 0).all() and torch.isnan(out[5:8]).all() and (out[8] == 0).all()
    c.check(out, rows=range(9, 14))


def test_attend_strided_rows_and_layers():
    c = Case("bf16", 8, 2, 128, 16, [40, 300], [5, 7], layers=3)
    B = binding()
    wide = torch.randn((12, 8 * 128 + 512), generator=c.g).to(torch.bfloat16)
    out = torch.full((12, 8 * 128 + 64), 7.0, dtype=torch.bfloat16, device="cuda")
    tab = torch.full((2, 64), -1, dtype=torch.int32)
    tab[:, :c.table.shape[1]] = c.table
    view = lambda t, at: t[:, at:at + 1024].unflatten(1, (8, 128))
    B.la_paged_tree_attend(B.la_pages(c.k.cuda(), c.v.cuda()), 2, view(wide.cuda(), 512), tab.cuda()[:, :c.table.shape[1]], i32(c.first), i32(c.lens), i64(c.vis), 7, view(out, 64))
    c.q = view(wide, 512)
    c.check(view(out, 64).cpu())
    assert (out[:, :64] == 7).all()


def test_attend_small_weights_beside_a_large_one():
    """Keys of 2^-25 times the first one's weight, 512 of them, whose V are what is left: half precision has no such numbers."""
    c = Case("f16", 1, 1, 64, 16, [513], [3], masks=[[1, 3, 5]])
    c.q[:] = 0
    c.q[:, :, 0] = 8.0
    for t in range(516):
        k, v = c.k[c.place(0, t)], c.v[c.place(0, t)]
        k[:], v[:] = 0, 1.0
        k[:, 0] = 0.0 if t == 0 else -2.166
        v[:] = 0.0 if t == 0 else 1.0
        c.keys[0][0][t], c.keys[0][1][t] = k, v
    out = c.run(scale=1.0)
    want = torch.softmax(torch.tensor([0.0] + [8.0 * float(torch.tensor(-2.166).half())] * 515, dtype=torch.float64), 0)[1:].sum()
    for i, n in ((0, 513), (1, 514), (2, 514)):
        mass = float(want) * n / 515
        # (the output, 1.5e-5, lies below 2^-14, where half precision's numbers are 2^-24 apart: rounding alone is off by up to 2^-25)
        assert (out[i].double() - mass).abs().max() <= 2.0 ** -10 * mass + 2.0 ** -25


def test_attend_a_pool_behind_32_bits():
    """Pages whose offsets pass 2^32 bytes, keys of them at both ends."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough memory")
    B = binding()
    n_pages = (5 << 30) // (16 * 8 * 128 * 2)
    k = torch.empty((1, n_pages, 8, 16, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    for heads, rows in ((8, 12), (32, 64)):
        c = Case("bf16", heads, 8, 128, 16, [600, 50, 2000], [rows, 3, 1])
        spots = torch.linspace(0, n_pages - 1, c.k.shape[1]).long()
        k[0, spots.cuda()], v[0, spots.cuda()] = c.k[0].cuda(), c.v[0].cuda()
        table = torch.where(c.table >= 0, spots[c.table.clamp(min=0).long()].to(torch.int32), c.table)
        out = torch.empty_like(c.q, device="cuda")
        B.la_paged_tree_attend(B.la_pages(k, v), 0, c.q.cuda(), table.cuda(), i32(c.first), i32(c.lens), i64(c.vis), rows, out)
        c.check(out.cpu())


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page,rows", [("bf16", 32, 8, 128, 16, 16), ("f16", 24, 2, 96, 8, 5), ("bf16", 4, 4, 64, 24, 40), ("f16", 4, 1, 256, 16, 9), ("bf16", 8, 8, 128, 32, 3)])
def test_attend_pages_of_a_pool_that_no_cache_holds(dtype, Hq, Hkv, dh, page, rows):
    """Pages of more than 256 MB a layer, most of them of nobody."""
    B = binding()
    c = Case(dtype, Hq, Hkv, dh, page, [600, 0, 2300], [rows, 3, rows - 1], seed=rows)
    n_pages = (150 << 20) // (page * Hkv * dh * 2)
    spots = torch.linspace(0, n_pages - 1, c.k.shape[1]).long()
    k, v = (torch.full((1, n_pages, Hkv, page, dh), float("nan"), dtype=T[dtype], device="cuda") for _ in range(2))
    k[0, spots.cuda()], v[0, spots.cuda()] = c.k[0].cuda(), c.v[0].cuda()
    table = torch.where(c.table >= 0, spots[c.table.clamp(min=0).long()].to(torch.int32), c.table)
    out = torch.empty_like(c.q, device="cuda")
    B.la_paged_tree_attend(B.la_pages(k, v), 0, c.q.cuda(), table.cuda(), i32(c.first), i32(c.lens), i64(c.vis), rows, out)
    c.check(out.cpu(), max_rows=rows)
    assert torch.equal(out.cpu(), c.run(max_rows=rows))


def test_attend_rows_of_one_are_the_paged_attentions():
    """A block of one row each is a decode step: as la_paged_attend's rows, within two roundings of the output."""
    B = binding()
    lens = [0, 5, 900, 3000]
    c = Case("bf16", 32, 8, 128, 16, lens, [1] * 4, masks=[[1]] * 4)
    out, pages = torch.empty_like(c.q, device="cuda"), B.la_pages(c.k.cuda(), c.v.cuda())
    B.la_paged_attend(pages, 0, c.q.cuda(), c.table.cuda(), None, i32(lens), out)
    assert (c.run(max_rows=1).double() - out.cpu().double()).abs().le(2.0 ** -7 * out.cpu().double().abs() + 1e-4).all()
