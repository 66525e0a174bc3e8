"""Adjusted logits of the rows of several requests' trees."""
import random

import pytest
import torch

from test_gpu_adjust import check, go
from test_gpu_tree import binding, i32, i64, random_tree

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("counts", [[5, 9, 1, 30], [64, 3], [12] * 5, [70, 2]])
def test_drafted_tokens_of_other_requests_do_not_count(counts):
    """With the masks that la_tree_layout leaves, a request's rows are what they are without the others', whatever those have drafted."""
    rng, V, R = random.Random(len(counts)), 400, len(counts)
    first, parent = [0], []
    for n in counts:
        parent += random_tree(rng, n)
        first.append(len(parent))
    N = len(parent)
    pos, vis = i32([0] * N), i64([0] * N)
    binding().la_tree_layout(i32(parent), i32(first), i32([3] * R), pos, vis)
    draft = [rng.randrange(V) for _ in range(N)]
    how = dict(R=R, req=[r for r, n in enumerate(counts) for _ in range(n)], rep=[1.3] * R, pres=[0.4] * R, freq=[0.2] * R, tokens=[[1, 2, 3]] * R, n_tokens=[3] * R, n_prompt=[1] * R, first=first,
               vis=[v % (1 << 64) for v in vis.tolist()], draft=draft)
    x = torch.randn((N, V), generator=torch.Generator().manual_seed(R)).cuda()
    got = go(x, **how)
    check(x, got, how)
    for r in range(R):
        mine = slice(first[r], first[r + 1])
        assert torch.equal(go(x, **dict(how, draft=[d if first[r] <= i < first[r + 1] else (d + 7) % V for i, d in enumerate(draft)]))[mine], got[mine])
