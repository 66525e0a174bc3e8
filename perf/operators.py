"""The operators of batched and sampled decoding, as cases to be timed and compared.

A case is one call of one operator:

  map     la_page_map: from the requests' lengths before and after a step, the pages they take and give
          back (block tables, ring of free pages) and of every new token its slot, position and request
  write   la_paged_write: K and V rows of new tokens into the pages of a layer
  attend  la_paged_attend: one query row per new token against the pages of its request, positions 0 .. pos
  logits  la_unembed_logits: final norm and unembedding, all logits stored
  sample  la_sample: temperature, top-k, top-p and min-p, one given random number per row

`run` has each in its plain form (elementary torch operations) and, where `own` is true, through the
library's public binding.  Widths are those of the repository's model shapes: 32 query heads on 8 of 128
channels, 4 on 2 of 64 in float32, heads 4096 x 32768 and 5120 x 131072.
"""
import math
import random

import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FLOAT_MAX = 3.4028234663852886e38
LEAST_WEIGHT = 2.0 ** -64  # (a token's weight relative to the largest one's; below it counts as none)


def listed():
    def attend(name, dtype, rows, Hq, Hkv, dh, page, ctx, spread):
        return {"name": name, "kind": "attend", "dtype": dtype, "rows": rows, "Hq": Hq, "Hkv": Hkv, "dh": dh, "page": page,
                "ctx": ctx, "spread": spread}

    return [
        # every decode step of a batch: each request grows by one token, a few of them into a new page
        {"name": "map_step_48", "kind": "map", "R": 48, "page": 16, "ctx": 4096, "rows": 48, "mode": "step"},
        # a scheduler's turn: new prompts, running requests, cropped and finished ones
        {"name": "map_turn_512", "kind": "map", "R": 512, "page": 32, "ctx": 32768, "rows": 400000, "mode": "turn"},
        # K and V of a decode step of 64 requests, one layer
        {"name": "write_step_64", "kind": "write", "dtype": "bf16", "n": 64, "Hkv": 8, "dh": 128, "page": 16, "pool": 16384},
        # K and V of a long prompt moving into pages
        {"name": "write_prompt_16000", "kind": "write", "dtype": "f16", "n": 16000, "Hkv": 8, "dh": 128, "page": 16, "pool": 32768},
        # one chat request in its first turn: latency
        attend("attend_1_at_500", "bf16", 1, 32, 8, 128, 16, 512, "even"),
        # an ordinary batch: ragged lengths, two rows of padding
        attend("attend_32_ragged_4096", "bf16", 32, 32, 8, 128, 16, 4096, "ragged"),
        # two long documents
        attend("attend_2_at_131000", "f16", 2, 32, 8, 128, 64, 131072, "even"),
        # the tiny fp32 decoder, a page size that no tile divides
        attend("attend_17_f32", "f32", 17, 4, 2, 64, 24, 1008, "ragged"),
        # the head of one sampled step of one request
        {"name": "logits_1_32768", "kind": "logits", "dtype": "bf16", "rows": 1, "d": 4096, "V": 32768},
        # the head of a full batch on the large vocabulary
        {"name": "logits_48_131072", "kind": "logits", "dtype": "bf16", "rows": 48, "d": 5120, "V": 131072},
        # the choice of one request's token, the usual filters
        {"name": "sample_1_32768", "kind": "sample", "rows": 1, "V": 32768, "mode": "usual"},
        # a full batch with a request's own settings in every row, some without any filter, some greedy
        {"name": "sample_64_131072", "kind": "sample", "rows": 64, "V": 131072, "mode": "mixed"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["map", "write", "attend", "attend", "logits", "sample", "sample"])
    page = rng.choice([16, 16, 32, 64, 128, 8, 24, 40])
    if kind == "map":
        mode = rng.choice(["step", "turn"])
        R = _log_int(rng, 1, 512)
        return {"kind": kind, "R": R, "page": page, "ctx": _log_int(rng, 256, 32768), "rows": R if mode == "step" else R * 780,
                "mode": mode}
    dtype, Hq, Hkv, dh = rng.choice([("bf16", 32, 8, 128), ("bf16", 8, 2, 128), ("bf16", 6, 2, 64), ("f16", 32, 8, 128), ("f16", 8, 8, 64),
                                     ("bf16", 24, 2, 96), ("f16", 16, 1, 256), ("f32", 4, 2, 64), ("f32", 6, 3, 80)])
    if kind == "write":
        n = _log_int(rng, 1, 16000)
        return {"kind": kind, "dtype": dtype, "n": n, "Hkv": Hkv, "dh": dh, "page": page, "pool": max(1024, 2 * n)}
    if kind == "attend":
        rows = _log_int(rng, 1, 64)
        most = 4096 * 32 * 8 * 128 * 2 // (rows * Hkv * dh * (4 if dtype == "f32" else 2))  # (the ordinary batch's bytes)
        return {"kind": kind, "dtype": dtype, "rows": rows, "Hq": Hq, "Hkv": Hkv, "dh": dh, "page": page,
                "ctx": _log_int(rng, 64, max(128, min(65536, most))), "spread": rng.choice(["even", "ragged"])}
    if kind == "logits":
        dtype, d, V = rng.choice([("bf16", 4096, 32768), ("bf16", 5120, 131072), ("f16", 4096, 32768), ("bf16", 512, 2048), ("f32", 256, 1024),
                                  ("bf16", 520, 5003)])
        return {"kind": kind, "dtype": dtype, "rows": rng.randint(1, 48 if V == 131072 else 64), "d": d, "V": V}
    return {"kind": kind, "rows": _log_int(rng, 1, 64), "V": _log_int(rng, 1000, 131072), "mode": rng.choice(["usual", "mixed", "open"])}


# ---- inputs -------------------------------------------------------------------------------------------
def _rng(case, seed):
    return random.Random("%s %d" % (sorted((k, v) for k, v in case.items() if k != "name"), seed))


def _gen(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(_rng(case, seed).getrandbits(60))
    return g


def _i32(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _normal(g, size, dtype, std=1.0):
    return torch.randn(size, generator=g, device="cuda", dtype=torch.float32).mul_(std).to(dtype)


def _positions(case, seed=None):
    """Last position that each row sees; the same for every seed but for their order."""
    rng = random.Random(17)
    n, ctx = case["rows"], case["ctx"]
    if case["spread"] == "even":
        pos = [ctx - 1 - (11 + 7 * r) % max(1, ctx // 40) for r in range(n)]
    else:  # from one token to the longest, every sixteenth row padding
        pos = [-1 if r % 16 == 15 else min(ctx - 1, int(round(math.exp(rng.uniform(0.0, math.log(ctx)))))) for r in range(n)]
        pos[0] = ctx - 1
        if n > 2:
            pos[1] = 0
    if seed is not None:
        _rng(case, seed).shuffle(pos)
    return pos


def _requests(case, seed=None):
    """Lengths before and after a step; `turn`: a quarter new prompts, an eighth cropped, an eighth finished, the rest grows by one."""
    rng = random.Random(23)
    ctx, old, new = case["ctx"], [], []
    room = case["rows"]
    for r in range(case["R"]):
        a = _log_int(rng, 1, ctx - 1)
        kind = r % 8 if case["mode"] == "turn" else 7
        if kind < 2:
            a, b = 0, _log_int(rng, 1, min(4096, ctx))
        elif kind == 2:
            b = a - min(a, rng.randint(0, 60))
        elif kind == 3:
            b = 0
        else:
            b = a + 1
        if max(0, b - a) > room:
            b = a + room
        room -= max(0, b - a)
        old.append(a)
        new.append(b)
    if seed is not None:
        both = list(zip(old, new))
        _rng(case, seed).shuffle(both)
        old, new = [a for a, _ in both], [b for _, b in both]
    return old, new


def _pages_of(length, page):
    return (length + page - 1) // page


def _sampling(case, seed):
    """Per row: temperature, top-k, top-p, min-p."""
    rng = _rng(case, seed)
    rows = []
    for r in range(case["rows"]):
        kind = {"usual": 0, "open": 1}.get(case["mode"], r % 6)
        if kind == 0:
            rows.append((rng.uniform(0.6, 1.0), rng.choice([20, 40, 50, 64]), rng.uniform(0.8, 0.98), rng.choice([0.0, 0.05])))
        elif kind == 1:
            rows.append((rng.uniform(0.8, 1.2), 0, 1.0, 0.0))
        elif kind == 2:
            rows.append((rng.uniform(0.7, 1.3), 0, rng.uniform(0.5, 0.99), 0.0))
        elif kind == 3:
            rows.append((rng.uniform(0.7, 1.5), 0, 1.0, rng.uniform(0.01, 0.2)))
        elif kind == 4:
            rows.append((0.0, 0, 1.0, 0.0))
        else:
            rows.append((rng.uniform(0.8, 2.0), _log_int(rng, 1, case["V"]), rng.uniform(0.9, 1.0), 0.0))
    return rows


class _Model:
    """A model handle that holds a head (one narrow layer without weights), freed with the state."""

    def __init__(self, case, g_final, unembed):
        from types import SimpleNamespace
        from paper_2602_16760_amd import binding as B
        self._free = B.la_free_model
        shape = SimpleNamespace(n_layers=1, d_model=case["d"], n_q_heads=1, n_kv_heads=1, head_dim=64, d_ffn=64, vocab=case["V"], rms_eps=1e-5,
                                rope_theta=1e4, dtype=case["dtype"])
        self.handle = B.la_init_model(shape, None, g_final, unembed)
        torch.cuda.synchronize()  # (the library has packed its own copy)

    def __del__(self):
        self._free(self.handle)


def prepare(case, seed):
    g, kind = _gen(case, seed), case["kind"]
    s = {"case": case}
    if kind == "map":
        old, new = _requests(case, seed)
        page = case["page"]
        blocks = _pages_of(case["ctx"], page)
        used = [_pages_of(a, page) for a in old]
        taken = sum(max(0, _pages_of(b, page) - u) for b, u in zip(new, used))
        n_pages = sum(used) + taken + taken // 4 + 16
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
        table = torch.full((case["R"], blocks), -1, dtype=torch.int32)
        at, host = 0, order.cpu()
        for r, u in enumerate(used):
            table[r, :u] = host[at:at + u]
            at += u
        ring = torch.cat((host[at:], torch.full((at,), -1, dtype=torch.int32)))  # free pages from the ring's head on
        turn = _rng(case, seed).randrange(n_pages)
        s.update(old=_i32(old), new=_i32(new), table=table.cuda(), ring=ring.roll(turn).cuda(), heads=_i32([turn, n_pages - at, 0, 0]),
                 heads_out=_i32([0, 0, 0, 0]), slot=_i32([0] * case["rows"]), pos=_i32([0] * case["rows"]), req=_i32([0] * case["rows"]),
                 first=_i32([0] * (case["R"] + 1)))
    elif kind == "write":
        dtype = DTYPES[case["dtype"]]
        n_pages = _pages_of(case["pool"], case["page"])
        shape = (1, n_pages, case["Hkv"], case["page"], case["dh"])
        rows = (case["n"], case["Hkv"], case["dh"])
        s.update(k_pages=torch.zeros(shape, dtype=dtype, device="cuda"), v_pages=torch.zeros(shape, dtype=dtype, device="cuda"), k=_normal(g, rows, dtype),
                 v=_normal(g, rows, dtype))
        # a prompt lies in whole pages in any order, a step's tokens anywhere
        if case["n"] > 512:
            pages = torch.randperm(n_pages, generator=g, device="cuda")
            i = torch.arange(case["n"], device="cuda")
            s["slot"] = (pages[i // case["page"]] * case["page"] + i % case["page"]).to(torch.int32)
        else:
            s["slot"] = torch.randperm(n_pages * case["page"], generator=g, device="cuda")[:case["n"]].to(torch.int32)
    elif kind == "attend":
        dtype = DTYPES[case["dtype"]]
        page, blocks = case["page"], _pages_of(case["ctx"], case["page"])
        pos = _positions(case, seed)
        used = [_pages_of(p + 1, page) for p in pos]
        n_pages = sum(used) + 3
        order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32).cpu()
        table = torch.full((case["rows"], blocks), -1, dtype=torch.int32)
        at = 0
        for r, u in enumerate(used):
            table[r, :u] = order[at:at + u]
            at += u
        shape = (1, n_pages, case["Hkv"], page, case["dh"])
        s.update(k_pages=_normal(g, shape, dtype), v_pages=_normal(g, shape, dtype), table=table.cuda(), pos=_i32(pos),
                 req=_i32(list(range(case["rows"]))), q=_normal(g, (case["rows"], case["Hq"], case["dh"]), dtype, 1.5))
        s["out"] = torch.empty_like(s["q"])
    elif kind == "logits":
        dtype = DTYPES[case["dtype"]]
        d, V = case["d"], case["V"]
        s.update(hidden=_normal(g, (case["rows"], d), torch.float32), gain=torch.rand(d, generator=g, device="cuda") + 0.5,
                 unembed=_normal(g, (d, V), dtype, 0.02), logits=torch.empty((case["rows"], V), dtype=torch.float32, device="cuda"))
        if own:
            s["model"] = _Model(case, s["gain"], s["unembed"])
    else:
        B, V = case["rows"], case["V"]
        x = _normal(g, (B, V), torch.float32, 2.0)
        x += 4.0 * (torch.rand((B, V), generator=g, device="cuda") < 20.0 / V)  # a few likely tokens
        x[:, torch.randperm(V, generator=g, device="cuda")[:V // 50]] = -math.inf  # tokens that a grammar forbids
        rows = _sampling(case, seed)
        s.update(x=x, u=torch.rand(B, generator=g, device="cuda"), temperature=torch.tensor([r[0] for r in rows], device="cuda"),
                 top_k=_i32([r[1] for r in rows]), top_p=torch.tensor([r[2] for r in rows], device="cuda"),
                 min_p=torch.tensor([r[3] for r in rows], device="cuda"), ids=_i32([0] * B), prob=torch.empty(B, device="cuda"))
    if own and kind in ("write", "attend"):
        from paper_2602_16760_amd import binding as B
        s["pages"] = B.la_pages(s["k_pages"], s["v_pages"])
    return s


# ---- the plain forms ----------------------------------------------------------------------------------
def _plain_map(s):
    case = s["case"]
    page, rows = case["page"], case["rows"]
    old, new, table, ring = s["old"].long(), s["new"].long(), s["table"], s["ring"].long()
    blocks, n_pages = table.shape[1], ring.shape[0]
    head, n_free = s["heads"][0].long(), s["heads"][1].long()
    add = (new - old).clamp(min=0)
    had, has = (old + page - 1) // page, (new + page - 1) // page
    take, give = (has - had).clamp(min=0), (had - has).clamp(min=0)
    ends, take_ends, give_ends = add.cumsum(0), take.cumsum(0), give.cumsum(0)
    first = torch.cat((ends.new_zeros(1), ends))
    j = torch.arange(blocks, device=old.device)[None]
    from_ring = (head + (take_ends - take - had)[:, None] + j) % n_pages
    grown = (j >= had[:, None]) & (j < has[:, None])
    to_ring = (head + n_free + (give_ends - give - has)[:, None] + j) % n_pages
    shrunk = (j >= has[:, None]) & (j < had[:, None])
    longer = torch.cat((ring, ring.new_zeros(1)))
    longer[torch.where(shrunk, to_ring, n_pages).flatten()] = table.long().flatten()
    table = torch.where(grown, ring[from_ring], table.long())
    i = torch.arange(rows, device=old.device)
    req = torch.searchsorted(ends, i, right=True)
    real = req < old.shape[0]
    r = req.clamp(max=old.shape[0] - 1)
    pos = old[r] + i - first[r]
    slot = table[r, (pos // page).clamp(max=blocks - 1)] * page + pos % page
    heads = torch.stack(((head + take_ends[-1]) % n_pages, n_free - take_ends[-1] + give_ends[-1], ends[-1], ends.new_zeros(())))
    none = torch.full_like(i, -1)
    out = (table, longer[:-1], heads, torch.where(real, slot, none), torch.where(real, pos, none), torch.where(real, req, none), first)
    return tuple(t.to(torch.int32) for t in out)


def _plain_write(s):
    page = s["case"]["page"]
    slot = s["slot"].long()
    for pages, rows in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
        pages[0, slot // page, :, slot % page] = rows
    return s["k_pages"], s["v_pages"]


def _plain_attend(s):
    case = s["case"]
    B, Hq, Hkv, dh = case["rows"], case["Hq"], case["Hkv"], case["dh"]
    table = s["table"][s["req"].long()].long().clamp(min=0)
    k = s["k_pages"][0][table].float().transpose(1, 2).reshape(B, Hkv, -1, dh)
    v = s["v_pages"][0][table].float().transpose(1, 2).reshape(B, Hkv, -1, dh)
    q = s["q"].float().view(B, Hkv, Hq // Hkv, dh)
    score = torch.matmul(q, k.transpose(2, 3).contiguous()) * dh ** -0.5
    seen = torch.arange(k.shape[2], device=k.device)[None] <= s["pos"].long()[:, None]
    score = torch.where(seen[:, None, None], score, -math.inf)
    top = score.amax(3, keepdim=True).clamp(min=-FLOAT_MAX)
    p = torch.exp(score - top)
    total = p.sum(3, keepdim=True)
    out = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return out.view(B, Hq, dh).to(s["q"].dtype)


def _plain_logits(s):
    h = s["hidden"]
    n = h / torch.sqrt((h * h).mean(1, keepdim=True) + 1e-5) * s["gain"]
    return torch.matmul(n, s["unembed"].float())


def _plain_sample(s):
    x = torch.where(torch.isnan(s["x"]), -math.inf, s["x"]).clamp(max=FLOAT_MAX).double()
    B, V = x.shape
    T, p, low, u = (s[n].double()[:, None] for n in ("temperature", "top_p", "min_p", "u"))
    k = torch.where(s["top_k"] > 0, s["top_k"], V).long()[:, None]
    value, order = torch.sort(x, dim=1, descending=True, stable=True)
    top, some = value[:, :1], value[:, :1] > -math.inf
    greedy = T <= 0
    w = torch.where(value > -math.inf, torch.exp((value - top) / torch.where(greedy, 1.0, T)), 0.0)
    w = torch.where(w < LEAST_WEIGHT, 0.0, w)
    rank = torch.arange(V, device=x.device)[None]
    in_k = torch.where(rank < k, w, 0.0)
    through = in_k.cumsum(1)
    before = torch.cat((torch.zeros_like(through[:, :1]), through[:, :-1]), 1)
    keep = (rank < k) & ((p >= 1) | (before < p * through[:, -1:])) & (w >= low) & (~greedy)
    keep[:, 0] = True
    w = torch.zeros_like(x).scatter_(1, order, torch.where(keep, w, 0.0))
    ends = w.cumsum(1)
    total = ends[:, -1:].contiguous()
    at = torch.minimum(torch.searchsorted(ends, u * total, right=True), torch.searchsorted(ends, total))
    prob = w.gather(1, at) / total
    ids = torch.where(some, torch.where(greedy, order[:, :1], at), -1)
    return ids[:, 0].to(torch.int32), torch.where(some, prob, 0.0)[:, 0].float()


def run(state):
    s, kind = state, state["case"]["kind"]
    if not own:
        return {"map": _plain_map, "write": _plain_write, "attend": _plain_attend, "logits": _plain_logits, "sample": _plain_sample}[kind](s)
    from paper_2602_16760_amd import binding as B
    if kind == "map":
        B.la_page_map(s["old"], s["new"], s["case"]["page"], s["table"], s["ring"], s["heads"], s["heads_out"], s["slot"], s["pos"], s["req"], s["first"])
        return s["table"], s["ring"], s["heads_out"], s["slot"], s["pos"], s["req"], s["first"]
    if kind == "write":
        B.la_paged_write(s["pages"], 0, s["k"], s["v"], s["slot"])
        return s["k_pages"], s["v_pages"]
    if kind == "attend":
        B.la_paged_attend(s["pages"], 0, s["q"], s["table"], s["req"], s["pos"], s["out"])
        return s["out"]
    if kind == "logits":
        B.la_unembed_logits(s["model"].handle, s["hidden"], s["logits"])
        return s["logits"]
    B.la_sample(s["x"], s["u"], s["ids"], s["prob"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
    return s["ids"], s["prob"]


# ---- what a pass cannot do without ----------------------------------------------------------------------
def work(case):
    kind, e = case["kind"], 4 if case.get("dtype") == "f32" else 2
    if kind == "map":
        old, new = _requests(case)
        moved = sum(abs(_pages_of(b, case["page"]) - _pages_of(a, case["page"])) for a, b in zip(old, new))
        return {"bytes": 12 * case["R"] + 8 * moved + 12 * case["rows"] + 36, "flops": 0}
    if kind == "write":
        return {"bytes": case["n"] * (4 * case["Hkv"] * case["dh"] * e + 4), "flops": 0}
    if kind == "attend":
        keys = sum(p + 1 for p in _positions(case))
        blocks = sum(_pages_of(p + 1, case["page"]) for p in _positions(case))
        return {"bytes": keys * case["Hkv"] * case["dh"] * 2 * e + 2 * case["rows"] * case["Hq"] * case["dh"] * e + 4 * blocks + 8 * case["rows"],
                "flops": 4 * keys * case["Hq"] * case["dh"]}
    if kind == "logits":
        d, V, n = case["d"], case["V"], case["rows"]
        return {"bytes": d * V * e + 4 * n * (d + V) + 4 * d, "flops": 2 * n * d * V}
    return {"bytes": 4 * case["rows"] * case["V"] + 28 * case["rows"], "flops": 4 * case["rows"] * case["V"]}


# ---- the definitions in 64 bits, written apart from the plain forms -----------------------------------------
def exact(case, seed):
    s, kind = prepare(case, seed), case["kind"]
    if kind == "map":
        return _exact_map(s)
    if kind == "write":
        out = []
        for pages, rows in ((s["k_pages"], s["k"]), (s["v_pages"], s["v"])):
            by_slot = pages[0].double().transpose(1, 2).reshape(-1, case["Hkv"], case["dh"])  # [page x place in it][head][channel]
            by_slot.index_copy_(0, s["slot"].long(), rows.double())
            out.append(by_slot.view(pages.shape[1], case["page"], case["Hkv"], case["dh"]).transpose(1, 2)[None].contiguous())
        return tuple(out)
    if kind == "attend":
        g = case["Hq"] // case["Hkv"]
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for b, last in enumerate(s["pos"].tolist()):
            if last < 0:
                continue
            at = torch.arange(last + 1, device="cuda")
            pages, place = s["table"][b].long()[at // case["page"]], at % case["page"]
            for h in range(case["Hkv"]):
                k, v = s["k_pages"][0, pages, h, place].double(), s["v_pages"][0, pages, h, place].double()
                q = s["q"][b, h * g:(h + 1) * g].double()
                out[b, h * g:(h + 1) * g] = torch.softmax(q @ k.t() / math.sqrt(case["dh"]), 1) @ v
        return out
    if kind == "logits":
        h = s["hidden"].double()
        a = h * s["gain"].double()
        out = torch.empty((case["rows"], case["V"]), dtype=torch.float64, device="cuda")
        for c in range(0, case["V"], 16384):
            out[:, c:c + 16384] = a @ s["unembed"][:, c:c + 16384].double()
        return out * torch.rsqrt(h.pow(2).sum(1, keepdim=True) / case["d"] + 1e-5)
    return _exact_sample(s)


def _exact_map(s):
    page = s["case"]["page"]
    table, ring, first = s["table"].tolist(), s["ring"].tolist(), [0]
    head, n_free, _, _ = s["heads"].tolist()
    tail, slot, pos, req = head + n_free, [], [], []
    for r, (a, b) in enumerate(zip(s["old"].tolist(), s["new"].tolist())):
        for block in range(_pages_of(a, page), _pages_of(b, page)):
            table[r][block] = ring[head % len(ring)]
            head, n_free = head + 1, n_free - 1
        for block in range(_pages_of(b, page), _pages_of(a, page)):
            ring[tail % len(ring)] = table[r][block]
            tail, n_free = tail + 1, n_free + 1
        for t in range(a, b):
            slot.append(table[r][t // page] * page + t % page)
            pos.append(t)
            req.append(r)
        first.append(len(slot))
    pad = [-1] * (s["case"]["rows"] - len(slot))
    return tuple(_i32(v) for v in (table, ring, [head % len(ring), n_free, len(slot), 0], slot + pad, pos + pad, req + pad, first))


def _exact_sample(s):
    import numpy as np
    x = s["x"].cpu().numpy().astype(np.float64)
    T, p, low, u = (s[n].cpu().numpy().astype(np.float64) for n in ("temperature", "top_p", "min_p", "u"))
    ids, probs = [], []
    for b in range(x.shape[0]):
        row = x[b]
        if T[b] <= 0:
            ids.append(int(np.argmax(row)))
            probs.append(1.0)
            continue
        order = np.lexsort((np.arange(len(row)), -row))
        order = order[row[order] > -np.inf]
        w = np.exp((row[order] - row[order[0]]) / T[b])
        n = len(w)
        k = int(s["top_k"][b])
        if k > 0:
            n = min(n, k)
        if p[b] < 1:
            sums = np.cumsum(w[:n])
            n = min(n, 1 + int(np.searchsorted(sums, p[b] * sums[-1])))
        n = min(n, int(np.sum(w >= max(low[b], LEAST_WEIGHT))))
        kept = np.sort(order[:n])
        w = np.exp((row[kept] - row[order[0]]) / T[b])
        sums = np.cumsum(w)
        i = min(int(np.searchsorted(sums, u[b] * sums[-1], side="right")), len(kept) - 1)
        ids.append(int(kept[i]))
        probs.append(w[i] / sums[-1])
    return _i32(ids), torch.tensor(probs, dtype=torch.float64, device="cuda")
