"""Sampling and stored logits on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
INF = float("inf")


def binding():
    from paper_2602_16760_amd import binding as B
    return B


def draw(row, temperature=1.0, k=0, p=1.0, low=0.0, u=0.5):
    """The definition: (id, probability) of one row, and how near u comes to the border of another token."""
    x = np.asarray(row, dtype=np.float64).copy()
    x[np.isnan(x)] = -np.inf
    x = np.minimum(x, np.finfo(np.float32).max)
    if not (x > -np.inf).any():
        return -1, 0.0, 1.0
    first = int(np.argmax(x))
    if not temperature > 0:
        return first, 1.0, 1.0
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    w = np.exp((x[order] - x[first]) / np.float64(temperature))
    n = len(w)
    if 0 < k < n:
        n = k
    if p < 1:
        n = min(n, 1 if not p > 0 else 1 + int(np.searchsorted(np.cumsum(w[:n]), p * w[:n].sum())))
    n = min(n, int((w >= max(min(low, 1.0) if low > 0 else 0.0, 2.0 ** -64)).sum()))
    kept = np.sort(order[:n])
    w = np.exp((x[kept] - x[first]) / np.float64(temperature))
    ends = np.cumsum(w)
    u = min(max(u, 0.0), 1.0) if u == u else 0.0
    i = min(int(np.searchsorted(ends, u * ends[-1], side="right")), len(kept) - 1)
    gap = np.abs(ends / ends[-1] - u).min()
    return int(kept[i]), w[i] / ends[-1], gap


def sample(x, u, temperature=None, k=None, p=None, low=None, u_index=None, dtype=None):
    B = binding()
    n = x.shape[0]
    dev = lambda v, t: None if v is None else torch.as_tensor(v, dtype=t).cuda()
    ids, prob = torch.full((n,), -9, dtype=torch.int32, device="cuda"), torch.full((n,), -9.0, device="cuda")
    f, i = torch.float32, torch.int32
    B.la_sample(x.cuda(), dev(u, f), ids, prob, temperature=dev(temperature, f), top_k=dev(k, i), top_p=dev(p, f), min_p=dev(low, f), u_index=dev(u_index, i))
    return ids.tolist(), prob.tolist()


def check(x, u, temperature=None, k=None, p=None, low=None, near=1e-9):
    """Ids are equal; a row whose u lies within 1e-9 of a border may go to either side (the weights keep 36 bits).  Probabilities to float's half step and 2^-35."""
    ids, prob = sample(x, u, temperature, k, p, low)
    at = lambda v, b, d: d if v is None else float(np.float32(v[b])) if not isinstance(d, int) else int(v[b])
    for b in range(x.shape[0]):
        want = draw(x[b].double().numpy(), at(temperature, b, 1.0), at(k, b, 0), at(p, b, 1.0), at(low, b, 0.0), float(np.float32(u[b])))
        if want[2] < near and ids[b] != want[0]:
            continue
        assert ids[b] == want[0], f"row {b}: {ids[b]}, not {want[0]} (u = {u[b]}, k = {k and k[b]}, p = {p and p[b]}, low = {low and low[b]}, T = {temperature and temperature[b]})"
        assert abs(prob[b] - want[1]) <= (2.0 ** -24 + 2.0 ** -35) * want[1] + 1e-37, f"row {b}: probability {prob[b]}, not {want[1]}"
    return ids


def rows_of(V, B, seed, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((B, V), generator=g) * spread
    return x, torch.rand(B, generator=g).tolist(), np.random.default_rng(seed)


@pytest.mark.parametrize("V", [1, 2, 63, 64, 65, 1000, 1024, 8191, 8192, 8193, 32768, 50257])
def test_without_filters(V):
    x, u, _ = rows_of(V, 9, V)
    check(x, u)
    check(x, u, temperature=[0.3, 0.7, 1.0, 1.5, 3.0, 50.0, 1e-3, 0.05, 1.0])


@pytest.mark.parametrize("V", [7, 1000, 8193, 32768, 131072])
@pytest.mark.parametrize("which", ["k", "p", "low", "kp", "all"])
def test_filters(V, which):
    x, u, g = rows_of(V, 12, V + len(which))
    x[:, g.permutation(V)[:V // 10]] = -INF
    some = lambda f: [f() for _ in range(12)]
    k = some(lambda: int(np.exp(g.uniform(0, np.log(1.2 * V))))) if "k" in which or which == "all" else None
    p = some(lambda: float(g.uniform(0.05, 1.0))) if "p" in which or which == "all" else None
    low = some(lambda: float(np.exp(g.uniform(-9, 0)))) if which in ("low", "all") else None
    if k:
        k[:4] = [1, 0, V, -3]
    if p:
        p[1:4] = [1.0, 0.0, 0.999999]
    if low:
        low[2:4] = [1.0, 0.0]
    check(x, u, some(lambda: float(g.uniform(0.4, 2.0))), k, p, low)


@pytest.mark.parametrize("dtype", ["bf16", "f16", "f32"])
def test_types_and_strides(dtype):
    """Many ties in the short types; rows that start anywhere."""
    x, u, g = rows_of(5003, 6, 5)
    wide = torch.full((6, 5003 + 4), 99.0)
    wide[:, 1:-3] = x
    x = wide.to(T[dtype])[:, 1:-3]
    B = binding()
    dev = wide.to(T[dtype]).cuda()[:, 1:-3]
    k, p = [0, 5, 40, 300, 2000, 5002], [0.9, 1.0, 0.5, 0.8, 0.97, 0.3]
    ids, prob = torch.zeros(6, dtype=torch.int32, device="cuda"), torch.zeros(6, device="cuda")
    B.la_sample(dev, torch.tensor(u).cuda(), ids, prob, top_k=torch.tensor(k, dtype=torch.int32).cuda(), top_p=torch.tensor(p).cuda())
    for b in range(6):
        want = draw(x[b].double().numpy(), 1.0, k[b], float(np.float32(p[b])), 0.0, float(np.float32(u[b])))
        assert int(ids[b]) == want[0] and abs(float(prob[b]) - want[1]) <= 2e-7 * want[1]


@pytest.mark.parametrize("V", [8, 100, 5000, 20000, 70000])
def test_equal_logits_share_equally(V):
    """Ties go by index: more of them than the list in LDS holds, borders hit exactly."""
    x = torch.full((8, V), -3.25)
    u = [0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 0.5, 0.5, 0.0]
    k = [0, 0, 0, 0, 0, 4, 0, V // 2]
    p = [1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 0.5, 0.25]
    ids = check(x, u, None, k, p, [0, 0, 0, 0, 0, 0, 0, 1.0], near=-1.0)
    assert ids[0] == 0 and ids[4] == V - 1 and ids[5] == 2


def test_two_values_and_many_ties():
    g = np.random.default_rng(4)
    x = torch.tensor(np.where(g.random((6, 30000)) < 0.3, 1.5, 1.4375), dtype=torch.float32)
    check(x, [0.1, 0.9, 0.33, 0.5, 0.77, 0.999], [1.0] * 6, [20000, 5000, 0, 0, 15000, 25000], [1.0, 0.7, 0.9, 0.2, 0.95, 1.0], [0, 0, 0, 0.95, 0, 0.5])


def test_ends_of_the_range():
    """Rows without a token, NaN, infinities, the type's lowest value, one token, extreme temperatures, u outside [0, 1)."""
    V = 9000
    g = torch.Generator().manual_seed(1)
    x = torch.randn((14, V), generator=g)
    x[0] = -INF
    x[1] = float("nan")
    x[2, 5:] = float("nan")
    x[3, 100] = x[3, 8500] = INF
    x[4] = torch.finfo(torch.float32).min
    x[5] = -INF
    x[5, 8999] = torch.finfo(torch.float32).min
    x[6] *= 1e30
    x[9] = x[9] * 0.0
    x[9, ::2] *= -1.0  # -0 and 0 are equal
    temp = [1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1.0, 1e-30, INF, 1.0, 0.0, -1.0, float("nan"), 1e30]
    u = [0.5, 0.5, 0.9, 0.75, 0.6, 0.3, 0.5, 0.5, 0.37, 0.7, 0.4, 0.4, 0.4, 0.123]
    ids = check(x, u, temp)
    assert ids[:2] == [-1, -1] and ids[3] == 8500 and ids[5] == 8999
    check(x, u, temp, k=[7] * 14, p=[0.8] * 14, low=[0.1] * 14)
    ids, _ = sample(x[7:10], [-1.0, 2.0, float("nan")])
    assert ids[0] == 0 and ids[1] == V - 1 and ids[2] == 0


def test_a_weight_below_2_to_the_minus_64_counts_as_none():
    x = torch.zeros((2, 10))
    x[:, 0], x[:, 3] = -45.0, -44.0  # exp(-45) is below 2^-64, exp(-44) above
    ids, prob = sample(x, [0.0, 0.0], k=[0, 9])
    assert ids == [1, 1] and all(abs(q - 0.125) < 1e-7 for q in prob)
    x[:, 1] = x[:, 2] = -INF
    assert sample(x, [0.0, 0.0])[0] == [3, 3]


def test_random_numbers_by_index():
    """Rows at one position draw with one number: equal rows give equal tokens.  An index outside is clamped."""
    x, _, _ = rows_of(4000, 5, 8)
    x[3] = x[1]
    u = torch.rand(30, generator=torch.Generator().manual_seed(2)).tolist()
    at = [4, 17, 9, 17, 29]
    ids, _ = sample(x, u, u_index=at)
    assert ids == [draw(x[b].double().numpy(), u=float(np.float32(u[a])))[0] for b, a in enumerate(at)] and ids[1] == ids[3]
    assert sample(x, u, u_index=[-5, 0, 29, 99, 3])[0][0] == sample(x, u, u_index=[0] * 5)[0][0]
    assert sample(x, u, u_index=[99] * 5)[0] == sample(x, u, u_index=[29] * 5)[0]


def test_a_row_does_not_depend_on_its_neighbours():
    x, u, g = rows_of(40000, 7, 21)
    p, k = [0.9, 1.0, 0.3, 0.99, 0.7, 1.0, 0.95], [0, 50, 20000, 3, 0, 0, 1000]
    ids, prob = sample(x, u, None, k, p)
    for b in range(7):
        assert sample(x[b:b + 1], u[b:b + 1], None, k[b:b + 1], p[b:b + 1]) == ([ids[b]], [prob[b]])


@pytest.mark.parametrize("filters", [{}, {"k": 6}, {"p": 0.8}, {"low": 0.1}])
def test_every_kept_token_is_drawn_as_often_as_it_weighs(filters):
    """4096 evenly spaced random numbers: a token of share s is drawn 4096 s times, up to one."""
    g = torch.Generator().manual_seed(3)
    row = torch.randn(50, generator=g) * 1.5
    n = 4096
    arg = {q: [v] * n for q, v in filters.items()}
    ids, prob = sample(row.repeat(n, 1), [(i + 0.5) / n for i in range(n)], **arg)
    count = np.bincount(ids, minlength=50)
    share = {i: q for i, q in zip(ids, prob)}
    assert abs(sum(share.values()) - 1) < 1e-5 + 1.0 / n * 50
    for i, q in share.items():
        assert abs(count[i] - n * q) <= 1.0 + 1e-3


# ---- stored logits ---------------------------------------------------------------------------------------
def head(d, V, dtype, seed=0):
    from types import SimpleNamespace
    B = binding()
    g = torch.Generator().manual_seed(seed)
    gain, un = torch.rand(d, generator=g) + 0.5, (torch.randn((d, V), generator=g) * 0.02).to(T[dtype])
    shape = SimpleNamespace(n_layers=1, d_model=d, n_q_heads=1, n_kv_heads=1, head_dim=64, d_ffn=64, vocab=V, rms_eps=1e-5, rope_theta=1e4, dtype=dtype)
    model = B.la_init_model(shape, None, gain.cuda(), un.cuda())
    torch.cuda.synchronize()
    return B, model, gain, un, g


def logits_of(h, gain, un):
    h = h.double()
    n = h * torch.rsqrt((h * h).mean(1, keepdim=True) + 1e-5) * gain.double()
    return n @ un.double(), n.abs() @ un.double().abs()


@pytest.mark.parametrize("d,V,dtype", [(256, 1024, "f32"), (520, 5003, "bf16"), (64, 16, "bf16"), (512, 2048, "bf16"), (384, 1536, "f16"), (1024, 5008, "bf16"),
                                       (8192, 272, "bf16"), (4096, 32768, "bf16"), (192, 36880, "f16")])
def test_logits(d, V, dtype):
    """Every row count's tiles, strided and unaligned rows.  Operands keep 2^-22 (two half-precision parts), weights 2^-25 absolutely (bfloat16 below 2^-14), sums are float:
    64 slices of at most d / 64 terms in a chain of d / 32 products."""
    B, model, gain, un, g = head(d, V, dtype)
    try:
        for n in (1, 15, 16, 17, 33, 48, 49, 64):
            h = torch.randn((n, d), generator=g) * 3.0
            for pad in (0, 1, 4):
                out = torch.full((n, V + pad), 7.0, device="cuda")
                B.la_unembed_logits(model, h.cuda(), out[:, pad:] if pad == 1 else out[:, :V])
                want, size = logits_of(h, gain, un)
                got = (out[:, pad:] if pad == 1 else out[:, :V]).cpu().double()
                norm = (h.double() * torch.rsqrt((h.double() ** 2).mean(1, keepdim=True)) * gain.double()).abs().sum(1, keepdim=True)
                tol = size * (d / 32 + 16) * 2.0 ** -24 + size * 2.0 ** -21 + (norm * 2.0 ** -25 if dtype == "bf16" else 0.0) + 1e-30
                assert ((got - want).abs() <= tol).all(), f"{n} rows: {float(((got - want).abs() / tol).max()):.2f} of the bound"
                assert pad == 0 or (out[:, 0 if pad == 1 else slice(V, None)] == 7).all()
                if d * V > 1 << 24:
                    break
    finally:
        B.la_free_model(model)


def test_logits_large_and_tiny_rows():
    """The norm takes the size out: 1e-3 and 1e4 of the same row, up to eps; half precision's range is in the norm's input."""
    B, model, gain, un, g = head(512, 2048, "bf16")
    try:
        h = torch.randn((1, 512), generator=g)
        rows = torch.cat((h * 1e4, h, h * 1e-3))
        out = torch.empty((3, 2048), device="cuda")
        B.la_unembed_logits(model, rows.cuda(), out)
        want, size = logits_of(rows, gain, un)
        assert ((out.cpu().double() - want).abs() <= size * 2.0 ** -18).all()
    finally:
        B.la_free_model(model)


@pytest.mark.parametrize("d,V,dtype", [(512, 2048, "bf16"), (384, 5008, "f16"), (256, 1024, "f32"), (520, 5003, "bf16")])
def test_logits_of_a_row_do_not_go_by_the_rows_beside_it(d, V, dtype):
    """Bit for bit, whatever tiles the other rows fill: what a sampled row draws rests on it."""
    B, model, _, _, g = head(d, V, dtype)
    try:
        h = (torch.randn((64, d), generator=g) * 2.0).cuda()
        all_, part = torch.empty((64, V), device="cuda"), torch.empty((64, V), device="cuda")
        B.la_unembed_logits(model, h, all_)
        for n in (1, 2, 15, 16, 17, 31, 33, 48, 49, 63):
            B.la_unembed_logits(model, h[64 - n:], part[:n])
            assert torch.equal(part[:n], all_[64 - n:]), f"{n} rows"
    finally:
        B.la_free_model(model)


@pytest.mark.parametrize("V", [64, 100, 5000, 20000])
@pytest.mark.parametrize("value", [-3.25, 1e30, -1e30, 1e-10, 7.3, -0.1])
def test_equal_logits_of_any_size_share_equally(V, value):
    """Where logit / temperature is so large that it has no fraction left, and where it has: a number on the border of two equal tokens' shares draws the one behind it, with and
    without filters that leave all of them.  (Sums of up to 2^14 equal weights of 37 bits are exact.)"""
    for temperature in (1.0, 1e-38, 1e-37, 1e-20, 1e-3):
        x, u = torch.full((9, V), value), [0.25, 0.5, 0.75] * 3
        k, low = [0, 0, 0, V, V, V, 0, 0, 0], [0.0] * 3 + [0.07] * 3 + [0.14] * 3
        ids, prob = sample(x, u, [temperature] * 9, k, [1.0] * 9, low)
        assert ids == [V // 4, V // 2, 3 * V // 4] * 3, (temperature, ids)
        assert all(abs(q * V - 1) <= 2.0 ** -24 for q in prob)
