"""Attention of trees whose scores are so large that float has no fractions left for them: a float's spacing at the score is many octaves of weight."""
import random

import pytest
import torch

from test_gpu_tree import Case, binding, i32

pytestmark = pytest.mark.gpu


def scores_of_one_channel(c, rng, a, b, rows):
    """Scores of one product each, which float holds exactly: rows of `a` times keys of `b`, in channel 0 alone; so keys of one b weigh the same."""
    total = c.lens[0] + rows
    ks = [rng.choice(b) for _ in range(total)]
    qs = [[rng.choice(a) for _ in range(c.Hq)] for _ in range(rows)]
    k = torch.zeros((total, c.Hkv, c.dh), dtype=c.dtype)
    k[:, :, 0] = torch.tensor(ks, dtype=torch.float64).to(c.dtype)[:, None]
    v = torch.randn((total, c.Hkv, c.dh), generator=c.g).to(c.dtype)
    for t in range(total):
        c.k[c.place(0, t)], c.v[c.place(0, t)] = k[t], v[t]
    c.q[:] = 0
    c.q[:, :, 0] = torch.tensor(qs, dtype=torch.float64).to(c.dtype)
    return k, v


@pytest.mark.parametrize("dtype,a,b", [
    ("f16", [20000.0, -17000.0, 40000.0], [20000.0, 19000.0, -21000.0, -20000.0, 3.0]), ("f16", [60000.0, -60000.0], [60000.0, -60000.0, 59000.0]), ("f16", [3000.0], [-3000.0, -2900.0]),
    ("f16", [1000.0, -900.0], [700.0, 650.0, -800.0, -750.0]), ("bf16", [3e6, -2e6], [1.0e6, 1.5e6, -1.25e6, 2.0]), ("bf16", [1e15, -1e15], [1e15, 2e15, -1e15, -3e15]),
    ("f32", [3e6, -2e6], [1.0e6, 1.5e6, -1.25e6, 2.0]), ("f32", [1e15], [-1e15, -3e15, -2e15])])
@pytest.mark.parametrize("rows,heads,dh,L,blocks", [(3, 2, 64, 300, None), (40, 2, 64, 300, None), (40, 4, 128, 2500, None), (60, 4, 64, 700, 1 << 14), (33, 2, 256, 1500, None), (1, 1, 80, 90, None)])
@pytest.mark.parametrize("scale", [1.0, -0.25])
def test_the_keys_of_the_largest_score_share_the_weight(dtype, a, b, rows, heads, dh, L, blocks, scale):
    """The next score below is so far away that its keys weigh nothing in 64 bits: the output is the mean of the V of the largest one's.  All of their weights are one number, of which 2^-20
    (bfloat16 2^-14) may be lost; the sums over n keys add 2^-23 a term, and the output is rounded by half a step."""
    rng = random.Random(rows + dh)
    c = Case(dtype, heads, 1, dh, 16, [L], [rows], masks=[[(2 << j) - 1 for j in range(rows)]], blocks=blocks)
    k, v = scores_of_one_channel(c, rng, a, b, rows)
    out = c.run(max_rows=rows, scale=scale)
    half = torch.finfo(c.dtype).eps / 2
    for j in range(rows):
        for h in range(heads):
            n = L + j + 1
            w = torch.softmax(k[:n, 0, 0].double() * float(c.q[j, h, 0]) * scale, 0)
            top = w == w.max()
            assert float(w[~top].sum()) < 2.0 ** -100 and float(w.max()) * int(top.sum()) == pytest.approx(1.0)
            want, mass = w @ v[:n, 0].double(), w @ v[:n, 0].double().abs()
            tol = (2.0 ** -14 if dtype == "bf16" else 2.0 ** -20) * mass + half * want.abs() + (n + 16) * 2.0 ** -23 * mass + torch.finfo(c.dtype).smallest_normal
            err = (out[j, h].double() - want).abs()
            assert (err <= tol).all(), f"row {j}, head {h}: {float((err / tol).nan_to_num(nan=float('inf')).max()):.2f} of the bound"


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,heads,dh,L", [(5, 2, 64, 100), (40, 2, 64, 100), (40, 4, 128, 1500), (20, 2, 256, 300), (6, 2, 80, 200)])
def test_a_row_whose_own_value_is_no_number(dtype, rows, heads, dh, L):
    """A drafted row that all but sees itself alone, its score of many products being far above the others', with an infinite V in one channel: the other channels are its own V, whatever the order
    in which float has added up its score.  The weight may lose 2^-20 (bfloat16 2^-14) and is divided by itself: a few steps of float, and half a step of the type."""
    c = Case(dtype, heads, 1, dh, 16, [L], [rows], masks=[[1 << j for j in range(rows)]])
    big = 2.0 ** 13 if dtype == "f16" else 2.0 ** 20
    half = torch.finfo(c.dtype).eps / 2
    k = (torch.randn((L + rows, 1, dh), generator=c.g) * big).to(c.dtype)
    k[:L] = 0
    v = torch.randn((L + rows, 1, dh), generator=c.g).to(c.dtype)
    v[L:, :, 3] = float("inf")
    for t in range(L + rows):
        c.k[c.place(0, t)], c.v[c.place(0, t)] = k[t], v[t]
    c.q[:] = k[L:]
    out = c.run(max_rows=rows, scale=1.0)
    others = [ch for ch in range(dh) if ch != 3]
    for j in range(rows):
        want = v[L + j].double().expand(heads, dh)
        assert (out[j, :, 3] == float("inf")).all()
        tol = ((2.0 ** -14 if dtype == "bf16" else 2.0 ** -20) + half + 32 * 2.0 ** -23) * want.abs() + torch.finfo(c.dtype).smallest_normal
        err = (out[j].double() - want).abs()
        assert (err[:, others] <= tol[:, others]).all(), f"row {j}: {float((err / tol)[:, others].nan_to_num(nan=float('inf')).max()):.2f} of the bound"


def test_scores_as_large_as_the_single_tokens_attention_takes():
    """A block of one row is a decode step: la_paged_attend's output of the same call."""
    B = binding()
    for dtype, size in (("f16", 20000.0), ("bf16", 1e12), ("f32", 1e12)):
        c = Case(dtype, 4, 2, 64, 16, [300, 2000], [1, 1], masks=[[1], [1]])
        g = torch.Generator().manual_seed(4)
        c.q = (torch.randint(1, 4, c.q.shape, generator=g) * size).to(c.dtype)
        c.k = torch.where(torch.isnan(c.k), c.k, (torch.randint(-3, 4, c.k.shape, generator=g) * size / 4).to(c.dtype))
        out = torch.empty_like(c.q, device="cuda")
        B.la_paged_attend(B.la_pages(c.k.cuda(), c.v.cuda()), 0, c.q.cuda(), c.table.cuda(), None, i32(c.lens), out, scale=1.0)
        got = c.run(max_rows=1, scale=1.0)
        assert torch.isfinite(got).all() and (got.double() - out.cpu().double()).abs().le(2.0 ** -7 * out.cpu().double().abs() + 1e-4).all()
