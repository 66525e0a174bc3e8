"""Adjusted logits on the GPU (penalties, biases, masks) against a plain implementation in 64 bits."""
import random

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


def by_hand(x, req, R, rep=None, pres=None, freq=None, tokens=None, n_tokens=None, n_prompt=None, draft=None, first=None, vis=None, bias=None, bias_token=None, allowed=None, index=None):
    """The published rules, row by row, in float64; and the sum of the magnitudes that met."""
    x = x.double().numpy().copy()
    size = np.abs(np.where(np.isfinite(x), x, 0))
    V = x.shape[1]
    on = lambda v, off, positive=False: off if v is None or not np.isfinite(v) or (positive and v <= 0) else v
    for b in range(len(x)):
        r = req[b] if req is not None else b
        if 0 <= r < R:
            rho, beta, alpha = on(rep and rep[r], 1.0, True), on(pres and pres[r], 0.0), on(freq and freq[r], 0.0)
            prompt, out = [], []
            if tokens is not None:
                n = max(0, min(n_tokens[r], len(tokens[r])))
                p = 0 if n_prompt is None else n_prompt[r]
                prompt = [t for i, t in enumerate(tokens[r][:n]) if i < p]
                out = [t for i, t in enumerate(tokens[r][:n]) if i >= p]
            if draft is not None:
                out = out + [draft[first[r] + j] for j in range(1, 64) if vis[b] >> j & 1 and 0 <= first[r] + j < len(x)]
            count = np.bincount([t for t in out if 0 <= t < V], minlength=V).astype(np.float64)
            seen = (count > 0) | (np.bincount([t for t in prompt if 0 <= t < V], minlength=V) > 0)
            with np.errstate(all="ignore"):
                x[b] = np.where(seen, np.where(x[b] > 0, x[b] / rho, x[b] * rho), x[b])
                x[b] = np.where(count > 0, x[b] - alpha * count - beta, x[b])
            size[b] = np.maximum(size[b], np.where(np.isfinite(x[b]), np.abs(x[b]), 0)) + abs(alpha) * count + abs(beta)
            if bias is not None:
                for t, f in zip(bias_token[r], bias[r]):
                    if 0 <= t < V:
                        x[b, t] += f
                        size[b, t] += abs(f) if np.isfinite(f) else 0
        if allowed is not None:
            m = index[b] if index is not None else b
            if 0 <= m < len(allowed):
                for v in range(V):
                    if not allowed[m][v >> 5] >> (v & 31) & 1:
                        x[b, v] = -np.inf
    return torch.from_numpy(x), torch.from_numpy(size)


def go(x, out=None, **how):
    """The call with plain lists."""
    f32 = lambda v: None if v is None else torch.tensor(v, dtype=torch.float32, device="cuda")
    ints = lambda v: None if v is None else i32(v)
    wrap = lambda v: None if v is None else torch.tensor(np.array(v, dtype=np.uint64).astype(np.uint32).astype(np.int64) - (np.array(v) >> 31 << 32), device="cuda").to(torch.int32)
    out = torch.empty_like(x) if out is None else out
    vis = how.get("vis")
    binding().la_logits_adjust(x, out, req=ints(how.get("req")), repetition=f32(how.get("rep")), presence=f32(how.get("pres")), frequency=f32(how.get("freq")), tokens=ints(how.get("tokens")),
                               n_tokens=ints(how.get("n_tokens")), n_prompt=ints(how.get("n_prompt")), draft=ints(how.get("draft")), first=ints(how.get("first")),
                               vis=None if vis is None else torch.tensor([v - (1 << 64) if v >> 63 else v for v in vis], dtype=torch.int64, device="cuda"),
                               bias=f32(how.get("bias")), bias_token=ints(how.get("bias_token")), allowed=wrap(how.get("allowed")), allowed_index=ints(how.get("index")), n_requests=how.get("R"))
    return out


def check(x, got, how):
    """Six float operations at most (2^-24 of what meets in each, the division among them), as many additions as a token has biases, and the rounding to the type."""
    req, R = how.get("req"), how["R"]
    rest = {k: v for k, v in how.items() if k not in ("req", "R")}
    want, size = by_hand(x.cpu(), req, R, **rest)
    got = got.cpu().double()
    n = 6 + max([0] + [max(row.count(t) for t in row) if row else 0 for row in how.get("bias_token") or []])
    half = torch.finfo(x.dtype).eps / 2
    finite = torch.isfinite(want)
    least = torch.finfo(x.dtype).smallest_normal * torch.finfo(x.dtype).eps
    tol = n * 2.0 ** -24 * size + half * want.abs() + least
    big = finite & (want.abs() + tol >= torch.finfo(x.dtype).max)  # (may round to an infinity)
    ok = torch.where(finite, (got - want).abs() <= tol, (got == want) | (torch.isnan(got) & torch.isnan(want))) | big
    assert ok.all(), f"{int((~ok).sum())} of {ok.numel()}, first {torch.nonzero(~ok)[0].tolist()}: {got[~ok][0]} for {want[~ok][0]}"


def make(rng, V, B, R, history=0, tree=False, n_bias=0, masks=0, req=True):
    how = dict(R=R, rep=[rng.choice([1.0, 1.2, 0.7]) for _ in range(R)], pres=[rng.choice([0.0, 0.6, -0.4]) for _ in range(R)], freq=[rng.choice([0.0, 0.3, -0.1]) for _ in range(R)])
    zipf = lambda n: [int(V * rng.random() ** 3) if rng.random() < 0.97 else rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31]) for _ in range(n)]
    if req:
        how["req"] = sorted(rng.choice([-1, R, 2 ** 31 - 1] + list(range(R)) * 3) if not tree else b * R // B for b in range(B))
    if history:
        how.update(tokens=[zipf(history) for _ in range(R)], n_tokens=[rng.choice([history, history // 2, 0, history + 5, -3]) for _ in range(R)],
                   n_prompt=[rng.choice([0, history // 3, history, -1]) for _ in range(R)])
    if tree:
        how["first"] = [next((b for b, q in enumerate(how["req"]) if q >= r), B) for r in range(R + 1)]
        how.update(draft=zipf(B), vis=[rng.getrandbits(64) if rng.random() < 0.2 else rng.getrandbits(max(1, B // R)) for _ in range(B)])
    if n_bias:
        how.update(bias=[[rng.gauss(0, 3) for _ in range(n_bias)] for _ in range(R)], bias_token=[[rng.randrange(V) if rng.random() < 0.9 else rng.choice([-1, V, 0]) for _ in range(n_bias)] for _ in range(R)])
    if masks:
        how.update(allowed=[[rng.choice([0, 0xffffffff, rng.getrandbits(32)]) for _ in range((V + 31) // 32)] for _ in range(masks)], index=[rng.randint(-1, masks) for _ in range(B)])
    return how


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,B,R,kw", [
    (1, 1, 1, dict(history=3)), (31, 4, 4, dict(history=100, n_bias=3, masks=2)), (32, 3, 2, dict(masks=3)), (1000, 6, 3, dict(history=500, n_bias=20, masks=2)),
    (8191, 2, 2, dict(history=64, tree=True)), (8193, 4, 2, dict(history=9000, tree=True, n_bias=7, masks=1)), (32768, 3, 3, dict(history=700, n_bias=300)), (40001, 2, 1, dict(n_bias=1, masks=5)),
    (300, 64, 5, dict(history=33, tree=True, n_bias=2))])
def test_adjust(dtype, V, B, R, kw):
    rng = random.Random(V + B)
    how = make(rng, V, B, R, **kw)
    x = (torch.randn((B, V), generator=torch.Generator().manual_seed(V)) * 3).to(T[dtype]).cuda()
    got = go(x, **how)
    check(x, got, how)
    assert torch.equal(got, go(x, **how))


def test_adjust_parts_alone_and_none():
    """Each part without the others, and none at all, which copies the bits."""
    rng = random.Random(5)
    how = make(rng, 5000, 4, 4, history=300, n_bias=9, masks=4, req=False)
    how["index"] = None
    x = torch.randn((4, 5000), generator=torch.Generator().manual_seed(1)).cuda()
    for keep in (("rep", "tokens", "n_tokens"), ("pres", "tokens", "n_tokens", "n_prompt"), ("freq", "tokens", "n_tokens", "n_prompt"), ("bias", "bias_token"), ("allowed",), ("rep", "pres"), ()):
        part = dict(R=4, **{k: how[k] for k in keep})
        check(x, go(x, **part), part)
    x[1, 7] = float("nan")
    assert torch.equal(go(x).view(torch.int32), x.view(torch.int32))
    assert torch.equal(go(x, rep=[1.0] * 4, tokens=how["tokens"], n_tokens=how["n_tokens"]).view(torch.int32), x.view(torch.int32))


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
def test_adjust_numbers_that_are_none(dtype):
    """Infinities and NaN among logits, settings and biases."""
    inf, nan = float("inf"), float("nan")
    x = torch.tensor([[inf, -inf, nan, 0.0, -0.0, 1.0, -2.0, 3.0] * 5] * 6).to(T[dtype]).cuda()
    how = dict(R=6, rep=[nan, 0.0, -1.0, inf, 1.5, 1e30], pres=[nan, inf, -inf, 0.5, 0.5, 0.0], freq=[0.1, nan, 0.1, -inf, 0.2, 0.0], tokens=[list(range(40)) + [3, 5]] * 6, n_tokens=[42] * 6,
               n_prompt=[8] * 6, bias=[[inf, -inf, nan, 2.0]] * 6, bias_token=[[20, 21, 22, 23]] * 6, allowed=[[0xffffff0f, 0xff]] * 6)
    check(x, go(x, **how), how)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,n_bias", [(1731, 300), (600, 1300), (3, 513), (10111, 512), (2049, 511), (8200, 1025)])
def test_adjust_more_biases_than_one_turn_takes(dtype, V, n_bias):
    """Lists longer than the threads of a workgroup, tokens that are in several parts of them, rows of odd lengths beside each other."""
    rng = random.Random(V)
    how = make(rng, V, 4, 3, history=150, n_bias=n_bias, masks=2)
    x = (torch.randn((4, V), generator=torch.Generator().manual_seed(V)) * 3).to(T[dtype]).cuda()
    got = go(x, **how)
    check(x, got, how)
    go(x, out=x, **how)
    assert torch.equal(x, got)


@pytest.mark.parametrize("dtype", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("V,pad,at", [(1000, 24, 0), (1000, 1, 0), (1000, 24, 3), (4099, 5, 1), (50000, 16, 8)])
def test_adjust_strides_alignment_and_in_place(dtype, V, pad, at):
    rng = random.Random(V)
    how = make(rng, V, 3, 3, history=200, n_bias=5, masks=2)
    wide = torch.randn((3, V + pad + at), generator=torch.Generator().manual_seed(2)).to(T[dtype]).cuda()
    view = lambda t: t[:, at:at + V]
    out = torch.full((3, V + 2 * pad + at), 7.0, dtype=T[dtype], device="cuda")
    want = go(view(wide).contiguous(), **how)
    go(view(wide), out=view(out), **how)
    assert torch.equal(view(out), want) and (out[:, :at] == 7).all() and (out[:, at + V:] == 7).all()
    check(view(wide), want, how)
    same = wide.clone()
    go(view(same), out=view(same), **how)
    assert torch.equal(view(same), want) and torch.equal(same[:, at + V:], wide[:, at + V:]) and torch.equal(same[:, :at], wide[:, :at])


def test_adjust_strided_lists():
    """Histories, biases and masks of a wider buffer; rows beside each other do not matter."""
    B, V = binding(), 3000
    rng = random.Random(8)
    how = make(rng, V, 4, 4, history=150, n_bias=11, masks=4, req=False)
    how["index"] = None
    x = torch.randn((4, V), generator=torch.Generator().manual_seed(3)).cuda()
    want = go(x, **how)
    check(x, want, how)

    def wide(t, n):
        w = torch.full((t.shape[0], t.shape[1] + n), 1, dtype=t.dtype, device="cuda")
        w[:, 1:1 + t.shape[1]] = t
        return w[:, 1:1 + t.shape[1]]

    f32 = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")
    masks = torch.tensor(how["allowed"], device="cuda")
    masks = torch.where(masks >= 1 << 31, masks - (1 << 32), masks).to(torch.int32)
    out = torch.empty_like(x)
    B.la_logits_adjust(x, out, repetition=f32(how["rep"]), presence=f32(how["pres"]), frequency=f32(how["freq"]), tokens=wide(i32(how["tokens"]), 7), n_tokens=i32(how["n_tokens"]),
                       n_prompt=i32(how["n_prompt"]), bias=wide(f32(how["bias"]), 3), bias_token=wide(i32(how["bias_token"]), 3), allowed=wide(masks, 2))
    assert torch.equal(out, want)
    for b in range(4):
        alone = torch.empty((1, V), device="cuda")
        B.la_logits_adjust(x[b:b + 1], alone, req=i32([b]), repetition=f32(how["rep"]), presence=f32(how["pres"]), frequency=f32(how["freq"]), tokens=i32(how["tokens"]),
                           n_tokens=i32(how["n_tokens"]), n_prompt=i32(how["n_prompt"]), bias=f32(how["bias"]), bias_token=i32(how["bias_token"]), allowed=masks, allowed_index=i32([b]))
        assert torch.equal(alone[0], want[b])


@pytest.mark.parametrize("n_bias", [300, 4096])
def test_adjust_a_token_with_many_biases(n_bias):
    """A token listed many times has the sum, added in the list's order, and the same bits every time."""
    rng = random.Random(n_bias)
    V = 10000
    how = dict(R=2, bias=[[rng.gauss(0, 1) for _ in range(n_bias)] for _ in range(2)], bias_token=[[rng.choice([5, 6, 9000, rng.randrange(V)]) for _ in range(n_bias)] for _ in range(2)])
    x = torch.randn((2, V), generator=torch.Generator().manual_seed(4)).cuda()
    got = go(x, **how)
    want = x.cpu().clone()
    for b in range(2):
        for t, f in zip(how["bias_token"][b], torch.tensor(how["bias"][b], dtype=torch.float32)):
            want[b, t] = want[b, t] + f
    assert torch.equal(got.cpu(), want)


def test_adjust_largest_sizes():
    """The widest vocabulary, a long history, in the last token's chunk too."""
    V = 1 << 19
    rng = random.Random(1)
    tokens = [[rng.randrange(V) for _ in range(30000)] + [V - 1] * 40000]
    how = dict(R=1, rep=[1.1], freq=[0.001], pres=[0.2], tokens=tokens, n_tokens=[70000], n_prompt=[100], allowed=[[0xffffffff] * (V // 32)], bias=[[1.5]], bias_token=[[V - 1]])
    x = torch.randn((1, V), generator=torch.Generator().manual_seed(5)).cuda()
    got = go(x, **how)
    how.pop("allowed")
    check(x, got, how)
