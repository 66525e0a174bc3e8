"""Attention of trees where weights span more than a 16-bit type does: small ones beside a large one."""
import pytest
import torch

from test_gpu_tree import Case

pytestmark = pytest.mark.gpu

# (rows, heads, head_dim, blocks of the table): 16 columns a workgroup, 64, 128 (a table of which one workgroup in 512 has many keys), heads of 256; whole and cut
FORMS = [(3, 1, 64, None), (40, 1, 64, None), (40, 4, 128, None), (40, 4, 64, 1 << 14), (33, 2, 256, None), (5, 2, 256, None), (3, 2, 80, None)]


@pytest.mark.parametrize("rows,heads,dh,blocks", FORMS)
@pytest.mark.parametrize("k0,size", [(1.9, 1000.0), (2.25, 1000.0), (2.4492, 1000.0), (2.5508, 1000.0), (2.6992, 1000.0), (2.9004, 30000.0), (3.0508, 30000.0)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_small_weights_with_large_values(dtype, k0, size, rows, heads, dh, blocks):
    """512 and more keys of 2^-22 to 2^-35 times the first one's weight, whose V are what is left, as normal numbers of the type.  A weight is off by 2^-20 of it (bfloat16 2^-14) or, in half
    precision, by 2^-40 of the largest; the scores are one product each, scaled and taken by an exponential in float (72 steps of 2^-24 of them allowed), the sums over n keys add 2^-23 a term,
    and the output is rounded by half a step."""
    L = 600
    c = Case(dtype, heads, 1, dh, 16, [L], [rows], masks=[[1 | 1 << j for j in range(rows)]], blocks=blocks)
    k = torch.zeros((L + rows, 1, dh), dtype=c.dtype)
    v = torch.rand((L + rows, 1, dh), generator=c.g).mul_(0.5).add_(0.5).mul_(size).to(c.dtype)
    k[1:, :, 0], v[0] = -k0, 0.0
    for t in range(L + rows):
        c.k[c.place(0, t)], c.v[c.place(0, t)] = k[t], v[t]
    c.q[:], c.q[:, :, 0] = 0, 8.0
    out = c.run(max_rows=rows, scale=1.0)
    score = 8.0 * float(k[1, 0, 0])
    half = torch.finfo(c.dtype).eps / 2
    for j in range(rows):
        see = list(range(L)) + sorted({L, L + j})
        w = torch.softmax(torch.tensor([0.0] + [score] * (len(see) - 1), dtype=torch.float64), 0)
        vs = v[see, 0].double()
        want = w @ vs
        weight = (2.0 ** -20 * want + 2.0 ** -40 * vs.sum(0)) if dtype == "f16" else 2.0 ** -14 * want
        tol = weight + half * want + 2 * 72 * 2.0 ** -24 * abs(score) * want + (len(see) + 16) * 2.0 ** -23 * want
        err = (out[j].double() - want).abs()
        assert (err <= tol).all(), f"row {j}: {float((err / tol).max()):.2f} of the bound"
