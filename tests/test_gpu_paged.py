"""The shared cache on the GPU: block tables and slot maps, rows into pages, attention over pages, each against a plain
implementation in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def binding():
    from paper_2602_16760_amd import binding as B
    return B


def i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


# ---- la_page_map ---------------------------------------------------------------------------------------
def map_by_hand(old, new, page, table, ring, head, n_free, max_rows):
    """The published rules, request by request; (error, ...) leaves everything as it was."""
    table, ring, n, blocks = [list(r) for r in table], list(ring), len(ring), len(table[0])
    up = lambda x: (x + page - 1) // page
    none = lambda e: (table, ring, [head, n_free, 0, e], [-1] * max_rows, [-1] * max_rows, [-1] * max_rows, [0] * (len(old) + 1))
    if not (0 <= head < n and 0 <= n_free <= n):
        return none(4)
    if any(x < 0 or x > blocks * page for x in old + new):
        return none(3)
    if sum(max(0, b - a) for a, b in zip(old, new)) > max_rows:
        return none(2)
    taken = sum(max(0, up(b) - up(a)) for a, b in zip(old, new))
    if taken > n_free:
        return none(1)
    slot, pos, req, first, at, tail = [], [], [], [0], head, head + n_free
    for r, (a, b) in enumerate(zip(old, new)):
        for k in range(up(a), up(b)):
            table[r][k] = ring[at % n]
            at += 1
        for k in range(up(b), up(a)):
            ring[tail % n] = table[r][k]
            tail += 1
        for t in range(a, b):
            slot.append(table[r][t // page] * page + t % page)
            pos.append(t)
            req.append(r)
        first.append(len(slot))
    pad = [-1] * (max_rows - len(slot))
    given = tail - head - n_free
    return table, ring, [(head + taken) % n, n_free - taken + given, len(slot), 0], slot + pad, pos + pad, req + pad, first


class Map:
    def __init__(self, R, page, blocks, n_pages, max_rows, seed=0, table_extra=0):
        g = np.random.default_rng(seed)
        self.page, self.max_rows = page, max_rows
        self.wide = torch.full((R, blocks + table_extra), -7, dtype=torch.int32, device="cuda")
        self.table = self.wide[:, :blocks]
        self.ring = i32(g.permutation(n_pages).tolist())
        self.heads = i32([0, n_pages, 0, 0])
        self.slot, self.pos, self.req, self.first = i32([5] * max_rows), i32([5] * max_rows), i32([5] * max_rows), i32([5] * (R + 1))
        self.hand = ([[-7] * blocks for _ in range(R)], self.ring.tolist(), 0, n_pages)

    def step(self, old, new):
        out = i32([9, 9, 9, 9])
        binding().la_page_map(i32(old), i32(new), self.page, self.table, self.ring, self.heads, out, self.slot, self.pos, self.req, self.first)
        want = map_by_hand(old, new, self.page, *self.hand, self.max_rows)
        got = [t.tolist() for t in (self.table, self.ring, out, self.slot, self.pos, self.req, self.first)]
        for name, a, b in zip(("table", "ring", "heads", "slot", "pos", "req", "first"), got, want):
            assert a == b, f"{name} of {old} -> {new}"
        self.heads = out
        self.hand = (want[0], want[1], want[2][0], want[2][1])
        return want[2][3]


@pytest.mark.parametrize("R,page", [(1, 16), (3, 1), (17, 8), (64, 16), (65, 40), (300, 32), (1500, 16)])
def test_map_over_many_turns(R, page):
    """Requests grow, shrink, end and begin again; the ring goes round several times.  More requests than a workgroup takes, and than
    it takes at its fewest."""
    g = np.random.default_rng(R)
    blocks = 9
    cap = blocks * page
    m = Map(R, page, blocks, max(blocks, R * blocks // 2), R * 2 * page + cap)
    old, errors = [0] * R, set()
    for turn in range(14):
        new = []
        for a in old:
            k = g.integers(6)
            new.append(int(min(cap, a + 1 if k < 2 else a + g.integers(0, 2 * page + 1) if k < 4 else a if k == 4 else g.integers(0, a + 1) if a else 0)))
        if turn % 5 == 4:
            new = [0 if g.integers(2) else b for b in new]
        e = m.step(old, new)
        errors.add(e)
        if e == 0:
            old = new
    assert 0 in errors
    assert m.step(old, [0] * R) == 0  # everybody ends: all pages are free, each once
    head, free = m.heads.tolist()[:2]
    n = m.ring.numel()
    assert free == n and sorted(m.ring.tolist()) == list(range(n))


def test_map_a_long_prompt_beside_steps():
    """More rows than a thread's eight: the rows' parts of the grid."""
    m = Map(20, 16, 4096, 9000, 70000)
    m.step([0] * 20, [1 + r for r in range(20)])
    assert m.step([1 + r for r in range(20)], [60000 if r == 7 else 2 + r for r in range(20)]) == 0


def test_map_table_rows_may_be_strided():
    m = Map(5, 4, 6, 40, 64, table_extra=3)
    assert m.step([0] * 5, [3, 24, 0, 9, 4]) == 0
    assert (m.wide[:, 6:] == -7).all()


@pytest.mark.parametrize("error,old,new,n_pages,max_rows,heads", [
    (1, [0, 0], [33, 40], 5, 100, None),             # three pages and three
    (2, [0, 0], [33, 40], 9, 72, None),
    (3, [0, 4], [1, -1], 9, 72, None),
    (3, [0, -4], [1, 1], 9, 72, None),
    (3, [0, 0], [1, 16 * 8 + 1], 99, 720, None),
    (4, [0, 0], [1, 1], 9, 72, [9, 4, 0, 0]),
    (4, [0, 0], [1, 1], 9, 72, [-1, 4, 0, 0]),
    (4, [0, 0], [1, 1], 9, 72, [0, 10, 0, 0]),
    (3, [2 ** 31 - 1, 0], [-2 ** 31, 1], 9, 72, None),
])
def test_map_errors_change_nothing(error, old, new, n_pages, max_rows, heads):
    m = Map(2, 16, 8, n_pages, max_rows)
    if heads:
        m.heads = i32(heads)
        m.hand = (*m.hand[:2], heads[0], heads[1])
    assert m.step(old, new) == error


# ---- la_paged_write ---------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("n,Hkv,dh,page", [(1, 1, 8, 1), (5, 2, 64, 16), (64, 8, 128, 16), (33, 3, 80, 7), (200, 1, 256, 64)])
def test_write(dtype, n, Hkv, dh, page):
    g = torch.Generator().manual_seed(n)
    n_pages, B = 2 * n // page + 3, binding()
    shape = (2, n_pages, Hkv, page, dh)
    k0, v0 = (torch.randn(shape, generator=g).to(T[dtype]) for _ in range(2))
    both = torch.randn((n, 3 * Hkv * dh + 8 * 8), generator=g).to(T[dtype])  # rows of a wider buffer
    dev = both.cuda()
    view = lambda t, at: t[:, at:at + Hkv * dh].unflatten(1, (Hkv, dh))
    slot = torch.randperm(n_pages * page, generator=g)[:n].to(torch.int32)
    if n > 4:
        slot[1], slot[3] = -1, n_pages * page  # skipped
    pages = B.la_pages(k0.cuda(), v0.cuda())
    B.la_paged_write(pages, 1, view(dev, 0), view(dev, Hkv * dh + 64 - 64 % 8), slot.cuda())
    for i, s in enumerate(slot.tolist()):
        if 0 <= s < n_pages * page:
            k0[1, s // page, :, s % page] = view(both, 0)[i]
            v0[1, s // page, :, s % page] = view(both, Hkv * dh + 64)[i]
    assert torch.equal(pages.k.cpu(), k0) and torch.equal(pages.v.cpu(), v0)


# ---- la_paged_attend -----------------------------------------------------------------------------------------
class Case:
    """Pages in any order, NaN wherever no request has a position; rows in any order of requests."""

    def __init__(self, dtype, Hq, Hkv, dh, page, lens, seed=0, spread=1.0, blocks=None, layers=1):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.Hq, self.Hkv, self.dh, self.page, self.lens = T[dtype], Hq, Hkv, dh, page, lens
        used = [(n + page - 1) // page for n in lens]
        n_pages = sum(used) + 2
        order = torch.randperm(n_pages, generator=g).tolist()
        blocks = blocks or max(1, max(used))
        self.table = torch.full((len(lens), blocks), -1, dtype=torch.int32)
        self.k, self.v = (torch.full((layers, n_pages, Hkv, page, dh), float("nan"), dtype=self.dtype) for _ in range(2))
        self.rows = []
        at = 0
        for r, n in enumerate(lens):
            mine = order[at:at + used[r]]
            at += used[r]
            self.table[r, :used[r]] = torch.tensor(mine, dtype=torch.int32)
            k, v = ((torch.randn((n, Hkv, dh), generator=g)).to(self.dtype) for _ in range(2))
            self.rows.append((k, v))
            for b, p in enumerate(mine):
                part = slice(b * page, min(n, (b + 1) * page))
                m = part.stop - part.start
                self.k[layers - 1, p, :, :m] = k[part].transpose(0, 1)
                self.v[layers - 1, p, :, :m] = v[part].transpose(0, 1)
        self.layer = layers - 1
        self.g = g
        self.spread = spread

    def queries(self, B):
        return (torch.randn((B, self.Hq, self.dh), generator=self.g) * self.spread).to(self.dtype)

    def run(self, q, req, pos, scale=None, stream=None):
        B = binding()
        pages = B.la_pages(self.k.cuda(), self.v.cuda())
        qd, out = q.cuda(), torch.full(q.shape, 77.0, dtype=self.dtype, device="cuda")
        B.la_paged_attend(pages, self.layer, qd, self.table.cuda(), None if req is None else i32(req), i32(pos), out, scale=scale)
        torch.cuda.synchronize()
        return out.cpu()

    def check(self, q, req, pos, out, scale=None):
        """Against float64.  A probability is rounded to the type (half a step: eps / 2 of it), as is the output; scores are sums of dh float products,
        their error shifts a probability by as much relatively, the exponential and the sums over n keys add 2^-23 a term."""
        scale = self.dh ** -0.5 if scale is None else scale
        half = torch.finfo(self.dtype).eps / 2
        g = self.Hq // self.Hkv
        for b, (r, p) in enumerate(zip(req if req is not None else range(len(pos)), pos)):
            if p < 0 or r < 0 or r >= len(self.lens):
                assert (out[b] == 0).all(), f"row {b} sees nothing"
                continue
            k, v = (t[:p + 1].double().repeat_interleave(g, 1) for t in self.rows[r])
            s = torch.einsum("hd,nhd->hn", q[b].double(), k) * scale
            size = torch.einsum("hd,nhd->hn", q[b].double().abs(), k.abs()).amax(1) * abs(scale)
            w = torch.softmax(s, 1)
            want, mass = torch.einsum("hn,nhd->hd", w, v), torch.einsum("hn,nhd->hd", w, v.abs())
            n = p + 1
            shift = ((self.dh + 8) * 2.0 ** -24 * size)[:, None]
            tol = (half if self.dtype != torch.float32 else 0.0) * mass + half * want.abs() + 2 * shift * mass + (n + 16) * 2.0 ** -23 * mass + 1e-30
            err = (out[b].double() - want).abs()
            assert (err <= tol).all(), f"row {b} (request {r}, {n} keys): {float((err / tol).max()):.2f} of the bound"


SHAPES = [("bf16", 32, 8, 128, 16), ("f16", 8, 2, 128, 16), ("bf16", 6, 2, 64, 32), ("f32", 4, 2, 64, 24), ("bf16", 24, 2, 96, 16), ("f16", 16, 1, 256, 16),
          ("bf16", 32, 1, 128, 8), ("bf16", 20, 1, 64, 5), ("f16", 3, 3, 8, 1), ("f32", 6, 3, 80, 16), ("f32", 5, 1, 256, 3), ("bf16", 2, 2, 200, 48), ("f16", 17, 1, 128, 64),
          ("bf16", 8, 1, 256, 33)]


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page", SHAPES)
def test_attend_short_and_long_rows(dtype, Hq, Hkv, dh, page):
    """One position, ends inside a page, a tile and a block, padding rows, an unknown request, several rows of one request."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 700, 0]
    c = Case(dtype, Hq, Hkv, dh, page, lens)
    req = [r for r, n in enumerate(lens) for _ in range(1) if n] + [11, 11, 3, 13, -1, 4]
    pos = [n - 1 for n in lens if n] + [0, 350, -1, 5, 5, -9]
    q = c.queries(len(req))
    c.check(q, req, pos, c.run(q, req, pos))


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page,lens", [
    ("bf16", 32, 8, 128, 16, [5000, 1, 900, 4096]), ("bf16", 8, 8, 64, 64, [20000]), ("f32", 4, 2, 64, 24, [3001, 40, 3000]), ("f16", 12, 1, 256, 16, [9000, 77]),
    ("bf16", 16, 2, 112, 20, [2500, 2501, 600]), ("f16", 40, 1, 128, 16, [3000, 800])])
def test_attend_rows_cut_into_items(dtype, Hq, Hkv, dh, page, lens):
    """Rows that several workgroups share and a second launch joins, beside rows of one."""
    c = Case(dtype, Hq, Hkv, dh, page, lens, seed=3, spread=2.0)
    req, pos = list(range(len(lens))) + [0], [n - 1 for n in lens] + [lens[0] // 2]
    q = c.queries(len(req))
    out = c.run(q, req, pos)
    c.check(q, req, pos, out)
    assert torch.equal(out, c.run(q, req, pos))


@pytest.mark.parametrize("B", [64, 65, 130])
def test_attend_many_rows(B):
    """More rows than a wave's lanes look up at once; without a row map."""
    lens = [1 + (37 * r) % 600 for r in range(B)]
    c = Case("bf16", 8, 2, 64, 16, lens, seed=B)
    q = c.queries(B)
    pos = [n - 1 for n in lens]
    c.check(q, None, pos, c.run(q, None, pos))


def test_attend_strided_rows_and_layers():
    c = Case("bf16", 8, 2, 128, 16, [40, 300], layers=3)
    B = binding()
    wide = torch.randn((2, 8 * 128 + 512), generator=c.g).to(torch.bfloat16)
    out = torch.full((2, 8 * 128 + 64), 7.0, dtype=torch.bfloat16, device="cuda")
    tab = torch.full((2, 64), -1, dtype=torch.int32)
    tab[:, :c.table.shape[1]] = c.table
    view = lambda t, at: t[:, at:at + 1024].unflatten(1, (8, 128))
    B.la_paged_attend(B.la_pages(c.k.cuda(), c.v.cuda()), 2, view(wide.cuda(), 512), tab.cuda()[:, :c.table.shape[1]], None, i32([39, 299]), view(out, 64))
    c.check(view(wide, 512), None, [39, 299], view(out, 64).cpu())
    assert (out[:, :64] == 7).all()


@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("bf16", 12), ("f32", 12)])
def test_attend_pages_that_are_none(dtype, page):
    """A position whose table entry names no page is not seen; a position behind the table's end is not either."""
    c = Case(dtype, 4, 2, 64, page, [100, 100])
    q = c.queries(2)
    c.table[0, 2], c.table[1, :] = -5, 1 << 20
    out = c.run(q, None, [99, 99])
    assert (out[1] == 0).all()
    keep = [t for t in range(100) if t // page != 2]
    c.rows[0] = tuple(t[keep] for t in c.rows[0])
    c.lens[0] = len(keep)
    c.check(q[:1], None, [len(keep) - 1], out[:1])
    c = Case(dtype, 4, 2, 64, page, [4 * page, 30])
    q = c.queries(2)
    c.check(q, None, [4 * page - 1, 29], c.run(q, None, [2 ** 31 - 1, 29]))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("scale", [0.0, -0.3, 8.0])
def test_attend_other_scales(dtype, scale):
    c = Case(dtype, 4, 1, 64, 16, [200, 33], seed=9)
    q = c.queries(2)
    c.check(q, None, [199, 32], c.run(q, None, [199, 32], scale), scale)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_attend_infinite_values_are_seen_where_they_stand(dtype):
    """An infinite V of a seen position reaches its channel alone; scores of -inf alone give zeros; a NaN among the seen keys gives NaN, beside rows that
    do not see it."""
    c = Case(dtype, 2, 1, 64, 16, [40, 20, 33, 8])
    q = c.queries(5)
    at = lambda r, t: (0, int(c.table[r, t // 16]), 0, t % 16)
    c.v[at(0, 39)][5] = float("inf")
    c.k[0, int(c.table[1, 0])], c.k[0, int(c.table[1, 1])] = float("-inf"), float("-inf")
    q[1] = q[1].abs() + 0.5
    c.k[at(2, 30)][3] = float("nan")
    out = c.run(q, [0, 1, 2, 3, 2], [39, 19, 32, 7, 29])
    assert torch.isinf(out[0, :, 5]).all() and torch.isfinite(out[0, :, :5]).all() and torch.isfinite(out[0, :, 6:]).all()
    assert (out[1] == 0).all() and torch.isnan(out[2]).all()
    c.check(q[3:4], [3], [7], out[3:4])
    c.check(q[4:], [2], [29], out[4:])


def test_attend_a_pool_behind_32_bits():
    """Pages whose offsets pass 2^32 bytes, keys of them at both ends."""
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough memory")
    B = binding()
    n_pages = (5 << 30) // (16 * 8 * 128 * 2)
    k = torch.empty((1, n_pages, 8, 16, 128), dtype=torch.bfloat16, device="cuda")
    v = torch.empty_like(k)
    c = Case("bf16", 8, 8, 128, 16, [600, 50])
    spots = torch.linspace(0, n_pages - 1, c.k.shape[1]).long().cuda()
    k[0, spots], v[0, spots] = c.k[0].cuda(), c.v[0].cuda()
    table = torch.where(c.table >= 0, spots.cpu()[c.table.clamp(min=0).long()].to(torch.int32), c.table)
    q = c.queries(2)
    out = torch.empty_like(q, device="cuda")
    B.la_paged_attend(B.la_pages(k, v), 0, q.cuda(), table.cuda(), None, i32([599, 49]), out)
    c.check(q, None, [599, 49], out.cpu())
    rows = torch.randn((2, 8, 128), generator=c.g).to(torch.bfloat16)
    B.la_paged_write(B.la_pages(k, v), 0, rows.cuda(), rows.cuda(), i32([n_pages * 16 - 1, (n_pages - 1) * 16]))
    assert torch.equal(k[0, -1, :, 15].cpu(), rows[0]) and torch.equal(v[0, -1, :, 0].cpu(), rows[1])


@pytest.mark.parametrize("heads,old,error", [([2, 8, 0, 0], [17, 0], 4), ([2, 8, 0, 0], [16, 0], 0), ([2, 9, 0, 0], [1, 0], 4)])
def test_map_gives_back_no_more_pages_than_are_out(heads, old, error):
    """A ring of 9 with 8 (or all) free takes back one (none): more would go where free pages stand."""
    B = binding()
    table, ring = i32([[5, 6], [7, 8]]), i32(list(range(9)))
    slot, pos, req, first, out = i32([3] * 4), i32([3] * 4), i32([3] * 4), i32([3] * 3), i32([9] * 4)
    B.la_page_map(i32(old), i32([0, 0]), 16, table, ring, i32(heads), out, slot, pos, req, first)
    assert out.tolist() == [heads[0], heads[1] + (1 if error == 0 else 0), 0, error]
    want = list(range(9))
    if error == 0:
        want[(heads[0] + heads[1]) % 9] = 5
    assert ring.tolist() == want and table.tolist() == [[5, 6], [7, 8]] and slot.tolist() == [-1] * 4 and first.tolist() == [0] * 3


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page,B,long", [("bf16", 8, 2, 64, 16, 65, 9000), ("f16", 4, 1, 128, 16, 300, 5000), ("f32", 2, 1, 64, 12, 1100, 2000), ("bf16", 4, 2, 96, 24, 2500, 700)])
def test_attend_rows_beyond_a_wave(dtype, Hq, Hkv, dh, page, B, long):
    """More rows than lanes, and than threads of a workgroup, of fewer requests, a long one among them, with padding rows and unknown requests."""
    lens = [long, 1, 16, 300, long // 3, 77, 150]
    c = Case(dtype, Hq, Hkv, dh, page, lens, seed=B)
    req = [r % 8 if r % 3 else 1 + r % 6 for r in range(B)]
    pos = [-1 if r % 13 == 5 else (lens[k] if k < 7 else 9) * (1 + r % 5) // 5 - 1 for r, k in enumerate(req)]
    q = c.queries(B)
    out = c.run(q, req, pos)
    c.check(q, req, pos, out)
    assert torch.equal(out, c.run(q, req, pos))


@pytest.mark.parametrize("B", [64, 3000])
def test_attend_many_rows_that_are_not_cut(B):
    c = Case("bf16", 4, 2, 64, 16, [512, 1, 100, 33], seed=B)
    req, pos = [r % 4 for r in range(B)], [[512, 1, 100, 33][r % 4] * (1 + r % 7) // 7 - 1 for r in range(B)]
    q = c.queries(B)
    c.check(q, req, pos, c.run(q, req, pos))


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page", SHAPES)
def test_attend_short_rows_in_a_wide_table(dtype, Hq, Hkv, dh, page):
    """The same lengths where the table has room for 5000 positions: rows may be cut, and most of them have one item."""
    lens = [1, 2, 15, 16, 17, 31, 32, 33, 127, 128, 129, 700, 1900, 0]
    c = Case(dtype, Hq, Hkv, dh, page, lens, seed=4, blocks=5000 // page + 1)
    req = [r for r, n in enumerate(lens) if n] + [11, 12, 3, 14, -1, 4]
    pos = [n - 1 for n in lens if n] + [0, 350, -1, 5, 5, -9]
    q = c.queries(len(req))
    c.check(q, req, pos, c.run(q, req, pos))


@pytest.mark.parametrize("blocks", [None, 400])
def test_attend_a_hundred_thousand_rows(blocks):
    """All rows of a request and position alike, the first, last and some between against 64 bits."""
    lens, B = [300, 1, 40, 17], 100001
    c = Case("f16", 2, 1, 8, 16, lens, seed=7, blocks=blocks)
    req = [r % 4 for r in range(B)]
    pos = [lens[r] - 1 for r in req]
    q = c.queries(4).repeat(B // 4 + 1, 1, 1)[:B]
    out = c.run(q, req, pos)
    c.check(q[:4], req[:4], pos[:4], out[:4])
    assert torch.equal(out, out[:4].repeat(B // 4 + 1, 1, 1)[:B])


@pytest.mark.parametrize("Hq,dh", [(1, 8), (3, 256)])
def test_attend_the_longest_row(Hq, dh):
    """A table of 2^31 - 16 positions, a few pages of it: at its ends, in its middle and around it, beside a short row."""
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("not enough memory")
    B, blocks, page = binding(), (1 << 27) - 1, 16
    g = torch.Generator().manual_seed(dh)
    k, v = (torch.randn((1, 6, 1, page, dh), generator=g).to(torch.bfloat16) for _ in range(2))
    q = torch.randn((2, Hq, dh), generator=g).to(torch.bfloat16)
    table = torch.full((2, blocks), -1, dtype=torch.int32, device="cuda")
    at = [0, 1 << 20, blocks // 2, blocks // 2 + 1, blocks - 2, blocks - 1]
    for p, b in enumerate(at):
        table[0, b] = (p + 2) % 6
    table[1, 0] = 4
    out = torch.empty_like(q, device="cuda")
    B.la_paged_attend(B.la_pages(k.cuda(), v.cuda()), 0, q.cuda(), table, None, i32([blocks * page - 1, 4]), out)
    pages = [(p + 2) % 6 for p in range(6)]
    keys = [k[0, pages, 0].reshape(-1, dh), k[0, 4, 0, :5]]
    values = [v[0, pages, 0].reshape(-1, dh), v[0, 4, 0, :5]]
    half = torch.finfo(torch.bfloat16).eps / 2
    for r in range(2):
        w = torch.softmax(q[r].double() @ keys[r].double().t() * dh ** -0.5, 1)
        want, mass = w @ values[r].double(), w @ values[r].double().abs()
        size = (q[r].double().abs() @ keys[r].double().abs().t()).amax(1, keepdim=True) * dh ** -0.5
        tol = half * mass + half * want.abs() + 2 * (dh + 8) * 2.0 ** -24 * size * mass + (len(keys[r]) + 16) * 2.0 ** -23 * mass + 1e-30
        assert ((out[r].cpu().double() - want).abs() <= tol).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("n", [33, 512, 5000])
@pytest.mark.parametrize("gap", [10, 18, 22.5, 23.5, 25.2, 30, 36])
def test_attend_one_key_far_above_the_others(dtype, n, gap):
    """A first key of 2^gap times the weight of every other one, whose values are zeros: the output is what the others leave beside it, n - 1 small weights that are not lost.  Equal
    values, so the error is that of the weights: half a step of the type each, of the output as much, and of the exponentials and their sums 2^-23 a term; of the first score three
    roundings of up to 38 at 2^-24 (1 / ln 2, the product, the difference)."""
    blocks, dh, far = (n + 15) // 16, 64, 2.0 ** 15
    B = binding()
    k = torch.zeros((1, blocks, 1, 16, dh), dtype=T[dtype], device="cuda")
    v = torch.full_like(k, far)
    k[0, 0, 0, 0, 0], v[0, 0, 0, 0] = gap * float(np.log(2)), 0
    q, out = torch.zeros((1, 4, dh), dtype=T[dtype], device="cuda"), torch.empty((1, 4, dh), dtype=T[dtype], device="cuda")
    q[..., 0] = 1
    B.la_paged_attend(B.la_pages(k, v), 0, q, torch.arange(blocks, dtype=torch.int32, device="cuda")[None], None, i32([n - 1]), out, scale=1.0)
    w = (n - 1) * float(np.exp(-float(k[0, 0, 0, 0, 0])))
    want, half = far * w / (1 + w), torch.finfo(T[dtype]).eps / 2
    least = 2.0 ** -25 if dtype == "f16" else 0.0  # (half a step of half precision below 2^-14)
    tol = (2 * half + (n + 16) * 2.0 ** -23 + 114 * 2.0 ** -24) * want + least
    assert (out.double() - want).abs().max() <= tol


@pytest.mark.parametrize("dtype,Hq,Hkv,dh,page", [s for s in SHAPES if s[0] != "f32"])
@pytest.mark.parametrize("spread,blocks", [(1.0, None), (3.0, 6000)])
def test_attend_rounds_its_output_and_little_else(dtype, Hq, Hkv, dh, page, spread, blocks):
    """16-bit types, rows that are cut and such that are not: beside the output's rounding, and what float scores, exponentials and sums leave, a weight is off by its second part's
    rounding alone: 3/2 steps of the first times half a step, 2^-20 of it (half precision; 2^-40 of the largest one at least) or 2^-14 (bfloat16)."""
    lens = [1, 2, 33, 129, 700, 1500]
    c = Case(dtype, Hq, Hkv, dh, page, lens, seed=21, spread=spread, blocks=blocks and blocks // page + 1)
    q, pos = c.queries(len(lens)), [n - 1 for n in lens]
    out = c.run(q, None, pos)
    half, part, least, g = torch.finfo(T[dtype]).eps / 2, 2.0 ** -20 if dtype == "f16" else 2.0 ** -14, 2.0 ** -40 if dtype == "f16" else 0.0, Hq // Hkv
    for b, n in enumerate(lens):
        k, v = (t.double().repeat_interleave(g, 1) for t in c.rows[b])
        s = torch.einsum("hd,nhd->hn", q[b].double(), k) * dh ** -0.5
        size = torch.einsum("hd,nhd->hn", q[b].double().abs(), k.abs()).amax(1) * dh ** -0.5
        w = torch.softmax(s, 1)
        want, mass = torch.einsum("hn,nhd->hd", w, v), torch.einsum("hn,nhd->hd", w, v.abs())
        shift = ((dh + 8) * 2.0 ** -24 * size)[:, None]
        tol = half * want.abs() + (1 + half) * (part + 2 * shift + (n + 16) * 2.0 ** -23) * mass + n * least * v.abs().amax(0) + 2.0 ** -25
        err = (out[b].double() - want).abs()
        assert (err <= tol).all(), f"row of {n}: {float((err / tol).max()):.2f} of the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("gap", [0, 5.5, 13, 20, 27])
def test_attend_an_infinite_value_of_any_weight(dtype, gap):
    """Keys of 2^-gap of the largest weight and about it, one of them with an infinite V of each sign: the output is infinite there, and nowhere a NaN."""
    n, dh = 96, 64
    g = torch.Generator().manual_seed(int(10 * gap))
    B = binding()
    k, v = torch.zeros((1, 6, 1, 16, dh), dtype=T[dtype]), torch.randn((1, 6, 1, 16, dh), generator=g).to(T[dtype])
    k[0, :, 0, :, 0] = (-(gap + torch.rand((6, 16), generator=g)) * float(np.log(2))).to(T[dtype])
    k[0, 0, 0, 0, 0] = 0
    for i, t in enumerate((1, 17, 40, 63, 64, 95)):
        v[0, t // 16, 0, t % 16, 8 * i + 3] = float("inf") if i % 2 else float("-inf")
    q, out = torch.zeros((1, 3, dh), dtype=T[dtype], device="cuda"), torch.empty((1, 3, dh), dtype=T[dtype], device="cuda")
    q[..., 0] = 1
    B.la_paged_attend(B.la_pages(k.cuda(), v.cuda()), 0, q, i32([[0, 1, 2, 3, 4, 5]]), None, i32([n - 1]), out, scale=1.0)
    at = [8 * i + 3 for i in range(6)]
    assert out[0, :, at].tolist() == [[float("inf") if i % 2 else float("-inf") for i in range(6)]] * 3
    rest = [d for d in range(dh) if d not in at]
    assert torch.isfinite(out[0][:, rest]).all()


def test_strides_of_dimensions_of_one_are_not_asked():
    """One row, one head, a table of one block, whatever strides the views have there: as their copies."""
    B, g = binding(), torch.Generator().manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=g).to(torch.bfloat16).cuda()
    pages, copy = (B.la_pages(torch.zeros((1, 4, 1, 16, 64), dtype=torch.bfloat16, device="cuda"), torch.zeros((1, 4, 1, 16, 64), dtype=torch.bfloat16, device="cuda")) for _ in range(2))
    k, v = rand(1, 5, 64).transpose(0, 1), rand(1, 5, 64).transpose(0, 1)  # [5, 1, 64], one head of stride 320
    slot = i32([16, 17, 18, 40, 63])
    B.la_paged_write(pages, 0, k, v, slot)
    B.la_paged_write(copy, 0, k.reshape(5, 64).clone().view(5, 1, 64), v.reshape(5, 64).clone().view(5, 1, 64), slot)
    assert torch.equal(pages.k, copy.k) and torch.equal(pages.v, copy.v) and pages.k.count_nonzero() > 0
    q = rand(2 * 64 + 3)[:128].as_strided((1, 2, 64), (131, 64, 1))  # one row of a buffer whose rows are not 16-byte aligned
    out, want = (torch.empty((1, 2, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    table = i32([[1, 0, 2]]).as_strided((1, 1), (3, 3))
    B.la_paged_attend(pages, 0, q, table, None, i32([2]), out)
    B.la_paged_attend(pages, 0, q.reshape(128).clone().view(1, 2, 64), i32([[1]]), None, i32([2]), want)
    assert torch.equal(out, want) and out.count_nonzero() > 0
    ids = i32([7, 7])
    B.la_sample(torch.zeros((2, 1), device="cuda").as_strided((2, 1), (1, 5)), torch.zeros(2, device="cuda"), ids)
    assert ids.tolist() == [0, 0]
