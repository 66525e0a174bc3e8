"""Drafted trees as programs use them: through a model's layers, in generation, captured and replayed, on several streams, refused."""
import random

import numpy as np
import pytest
import torch

import synth
from gpu_util import gpu_engine, launch_names, oracle_model, row_rel_err
from oracle import transformer as otf
from test_gpu_tree import paths, random_tree

pytestmark = pytest.mark.gpu
BAR = {"f32": 1e-4, "bf16": 2e-2, "f16": 2e-3}
T = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def binding():
    from paper_2602_16760_amd import binding as B
    return B


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def i64(values):
    return torch.tensor([v - (1 << 64) if v >> 63 else v for v in values], dtype=torch.int64, device="cuda")


def bits(a, dtype):
    """numpy rows of synth -> torch rows of the pages' type."""
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.view(torch.bfloat16) if dtype == "bf16" and t.dtype != torch.float32 else t.to(T[dtype])


# ---- through the layers ---------------------------------------------------------------------------------
@pytest.mark.parametrize("name,lens,counts,page,env", [
    ("tiny_f32", [0, 5, 47, 300], [3, 0, 12, 7], 16, {}), ("small_bf16", [0, 31, 33, 700], [9, 1, 16, 5], 16, {}), ("small_bf16", [40], [64], 32, {}),
    ("small_bf16", list(range(3, 19)), [4] * 16, 24, {}), ("small64_bf16", [100, 2], [30, 20], 8, {}), ("small_f16", [64, 12, 1000], [20, 3, 33], 32, {}), ("small64_f16", [7] * 17, [3] * 17, 16, {}),
    ("small_bf16", [0, 40, 600], [5, 12, 8], 16, {"LA_FORCE_GENERIC": "1"}), ("small64_f16", [5, 90, 1], [6, 40, 2], 12, {"LA_FORCE_GENERIC": "1"}),
    ("small_bf16", [3, 33], [7, 9], 16, {"LA_WGS": "37"})])
def test_forward_against_the_oracle(name, lens, counts, page, env, monkeypatch):
    """Blocks of trees of several requests in one call: hidden states against the oracle's block of each request, K and V where the slots say, rows that hang on nothing and rows of no request
    among them."""
    for key, value in env.items():
        monkeypatch.setenv(key, value)
    shape = synth.SHAPES[name]
    eng, om, B = gpu_engine(shape, 64, head=False), oracle_model(shape, head=False), binding()
    R, H, dh, dt, rng = len(lens), shape.n_kv_heads, shape.head_dim, shape.dtype, random.Random(4)
    try:
        used = [(n + c + page - 1) // page for n, c in zip(lens, counts)]
        order = np.random.default_rng(2).permutation(sum(used))
        table = np.full((R, max(used)), -1, dtype=np.int32)
        k = torch.full((shape.n_layers, sum(used), H, page, dh), float("nan"), dtype=bits(np.zeros(1, np.float32), dt).dtype)
        v, at, rows = torch.full_like(k, float("nan")), 0, []
        first, trees, slot, pos, vis = [0], [], [], [], []
        for r, (n, c) in enumerate(zip(lens, counts)):
            u = used[r]
            table[r, :u] = order[at:at + u]
            at += u
            okv = otf.KVCache(shape, n + c)
            for l in range(shape.n_layers):
                if n:
                    kk, vv = synth.kv_fill(shape, l, n, r)
                    okv.fill(l, kk, vv)
                    for dst, src in ((k, bits(kk, dt)), (v, bits(vv, dt))):
                        for b in range((n + page - 1) // page):
                            part = src[b * page:(b + 1) * page]
                            dst[l, table[r, b], :, :len(part)] = part.transpose(0, 1)
            okv.L = n
            rows.append(okv)
            tree = paths([-1] + [p for p in random_tree(rng, c)[1:]]) if c else []
            trees.append(tree)
            pos += [n + d if m else -1 for d, m in tree]
            vis += [m for _, m in tree]
            slot += [int(table[r, (n + j) // page]) * page + (n + j) % page for j in range(c)]
            first.append(first[-1] + c)
        N = min(64, first[-1] + 2)
        pad = N - first[-1]
        x = synth.hidden_block(shape, N, 0)
        pages = B.la_pages(k.cuda(), v.cuda())
        args = (i32(pos + [-1] * pad), i64(vis + [0] * pad), i32(slot + [-1] * pad), i32(first), i32(lens), max(counts), pages, i32(table.tolist()))
        hidden = torch.from_numpy(x.astype(np.float32)).cuda()
        again = hidden.clone()
        run = lambda h: B.la_forward_tree(eng.model, 0, shape.n_layers, h, *args)
        used_names = launch_names(lambda: run(hidden.clone()))
        assert "tree_attend" in used_names and "paged_attend" not in used_names and ("pf_gemm_qkv" in used_names) == (dt != "f32" and "LA_FORCE_GENERIC" not in env), used_names
        run(hidden)
        run(again)
        assert torch.equal(again.nan_to_num(), hidden.nan_to_num())
        got = hidden.cpu().numpy()
        for r, (n, c) in enumerate(zip(lens, counts)):
            if not c:
                continue
            mine = range(first[r], first[r + 1])
            safe = [m if m else 1 << j for j, (_, m) in enumerate(trees[r])]  # (the oracle's rows see themselves at least; those of no use are not compared)
            want = otf.forward_block(om, rows[r], x[list(mine)], [n + max(d, 0) for d, _ in trees[r]], safe)
            there = [j for j, (_, m) in enumerate(trees[r]) if m]
            err = row_rel_err(got[list(mine)][there], want[there]).max()
            assert err <= BAR[dt], f"request {r} of {n} positions and {c} rows: {err:.2e}"
            for j in there:
                p, place = slot[first[r] + j] // page, slot[first[r] + j] % page
                for cache, theirs in ((pages.k, rows[r].K), (pages.v, rows[r].V)):
                    row = cache[shape.n_layers - 1, p, :, place].float().cpu().numpy()
                    ref = np.asarray(theirs[shape.n_layers - 1][n + j], dtype=np.float64).reshape(H, dh)
                    assert np.abs(row - ref).max() <= (BAR[dt] + 2.0 ** -8) * np.abs(ref).max()
    finally:
        eng.close()


def test_forward_in_ranges_of_layers():
    shape = synth.SHAPES["small_bf16"]
    eng, B = gpu_engine(shape, 64, head=False), binding()
    try:
        mk = lambda: B.la_pages(*(torch.zeros((3, 6, 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        table, first, lens = i32([[4, 2], [1, 0]]), i32([0, 4, 7]), i32([0, 0])
        pos, vis, slot = i32([0, 1, 1, 2, 0, 1, 2]), i64([1, 3, 5, 13, 1, 3, 7]), i32([64, 65, 66, 67, 16, 17, 18])
        x = torch.from_numpy(synth.hidden_block(shape, 7, 1).astype(np.float32)).cuda()
        a, b, pa, pb = x.clone(), x.clone(), mk(), mk()
        B.la_forward_tree(eng.model, 0, 3, a, pos, vis, slot, first, lens, 4, pa, table)
        for l in range(3):
            B.la_forward_tree(eng.model, l, l + 1, b, pos, vis, slot, first, lens, 4, pb, table)
        assert torch.equal(pa.k, pb.k) and torch.equal(pa.v, pb.v) and torch.equal(a, b)
        B.la_forward_tree(eng.model, 1, 1, b, pos, vis, slot, first, lens, 4, pb, table)
        assert torch.equal(a, b)
    finally:
        eng.close()


# ---- generation -------------------------------------------------------------------------------------------
def drafts_of(truth, prompts, vocab, seed, wrong=0.3):
    """Trees around the continuation that sequential generation found: some of its tokens, some others beside and behind them, some that hang on nothing."""
    rng = random.Random(seed)

    def draft(texts):
        out = []
        for r, text in enumerate(texts):
            if text is None:
                out.append(None if rng.random() < 0.5 else ([1, 2], [0, 1]))
                continue
            ahead = truth[r][len(text) - len(prompts[r]):]
            tokens, parents, tip = [], [], 0
            for t in ahead[:rng.randint(0, 6)]:
                for _ in range(rng.randint(0, 2)):  # (a sibling in front: other indexes for the path)
                    tokens.append(rng.randrange(vocab))
                    parents.append(rng.choice([tip, 0, -1, len(tokens)]))
                tokens.append(int(t) if rng.random() > wrong else rng.randrange(vocab))
                parents.append(tip)
                tip = len(tokens)
            out.append((tokens, parents))
        return out

    return draft


@pytest.mark.parametrize("sampling", [None, dict(temperature=0.8, top_k=30, top_p=0.9, seed=3), dict(temperature=0.7, seed=4, repetition=1.3, presence=0.4, frequency=0.2, bias={5: 2.0, 7: -3.0, 11: 1.0})])
@pytest.mark.parametrize("max_rows,page", [(16, 16), (5, 8), (1, 16), (64, 24)])
def test_trees_emit_what_sequential_generation_emits(sampling, max_rows, page):
    """The tiny decoder's rounding is far below its margins: with any drafts the tokens are the batch's, in fewer steps where drafts are right, and all pages come back."""
    shape = synth.SHAPES["tiny_f32"]
    eng = gpu_engine(shape, 200, seed=2)
    prompts = [np.random.default_rng(6).integers(0, shape.vocab, size=n).astype(np.int32) for n in (5, 40, 23)]
    try:
        want, _ = eng.generate_batch(prompts, 24, page_size=page, sampling=sampling)
        for wrong in (0.0, 0.4, 1.0):
            got, st = eng.generate_tree(prompts, 24, drafts_of(want, prompts, shape.vocab, 7, wrong), max_rows=max_rows, page_size=page, sampling=sampling)
            assert np.array_equal(got, want)
            assert st["free_pages"] == st["pages"] and st["steps"] <= 24
            assert max_rows == 1 or wrong > 0.0 or st["steps"] < 20
        one, st = eng.generate_tree(prompts[:1], 24, lambda texts: [([], [])], sampling=None if sampling is None else dict(sampling, u=_row(sampling, 24, 3, 0)))
        assert np.array_equal(one[0], want[0]) and st["steps"] == 24
    finally:
        eng.close()


def _row(sampling, n, R, r):
    """The random numbers of request r of R."""
    u = torch.rand(n * R, generator=torch.Generator(device="cuda").manual_seed(sampling.get("seed", 0)), device="cuda")
    return u.view(n, R)[:, r].clone()


def test_trees_of_a_16_bit_model_against_the_oracle():
    """Every emitted token is the oracle's choice behind the tokens in front of it, wherever its margin is clear."""
    shape = synth.SHAPES["small_bf16"]
    eng, om = gpu_engine(shape, 300, seed=1), oracle_model(shape, seed=1)
    prompts = [np.random.default_rng(5).integers(0, shape.vocab, size=n).astype(np.int32) for n in (1, 9, 90)]
    try:
        plain, _ = eng.generate_batch(prompts, 20)
        tokens, st = eng.generate_tree(prompts, 20, drafts_of(plain, prompts, shape.vocab, 2, 0.1), max_rows=21)
        assert st["free_pages"] == st["pages"] and st["steps"] < 20
        safe = 0
        for p, t in zip(prompts, tokens):
            logits = otf.causal_forward(om, np.concatenate([p, t]).astype(np.int64)[:-1])[1][len(p) - 1:]
            t1, t2 = otf.top2_margin(logits)
            clear = (t1 - t2) > 3e-2
            assert np.array_equal(otf.argmax_ids(logits)[clear], t[clear])
            safe += int(clear.sum())
        assert safe >= 20
    finally:
        eng.close()


def test_penalties_are_about_the_requests_own_tokens():
    """Greedy generation with penalties and biases: every token is the largest of the oracle's logits after the published rules, wherever its margin is clear."""
    shape = synth.SHAPES["tiny_f32"]
    eng, om = gpu_engine(shape, 200, seed=2), oracle_model(shape, seed=2)
    prompts = [np.random.default_rng(8).integers(0, shape.vocab, size=n).astype(np.int32) for n in (30, 4)]
    how, safe = dict(temperature=0.0, repetition=1.5, presence=0.05, frequency=0.02, bias={3: 0.1, 900: -0.5}), 0
    try:
        tokens, _ = eng.generate_batch(prompts, 20, sampling=how)
        plain, _ = eng.generate_batch(prompts, 20)
        assert not np.array_equal(tokens, plain)
        for p, t in zip(prompts, tokens):
            seq = np.concatenate([p, t]).astype(np.int64)
            logits = otf.causal_forward(om, seq[:-1])[1][len(p) - 1:].astype(np.float64)
            for i, x in enumerate(logits):
                seen, new = np.unique(seq[:len(p) + i]), np.bincount(t[:i], minlength=shape.vocab)
                x[seen] = np.where(x[seen] > 0, x[seen] / 1.5, x[seen] * 1.5)
                x -= 0.02 * new + 0.05 * (new > 0)
                x[3] += 0.1
                x[900] -= 0.5
                best = np.sort(x)[-2:]
                if best[1] - best[0] > 1e-3:
                    safe += 1
                    assert int(np.argmax(x)) == t[i]
        assert safe >= 30
    finally:
        eng.close()


def test_drafts_and_parameters_are_checked():
    eng = gpu_engine(synth.SHAPES["tiny_f32"], 64)
    p = [np.array([1, 2, 3])]
    try:
        for bad in (lambda: eng.generate_tree(p, 4, lambda t: [([1, 2], [0])]), lambda: eng.generate_tree(p, 4, lambda t: [None], max_rows=65), lambda: eng.generate_tree([], 4, lambda t: []),
                    lambda: eng.generate_tree(p, 4, lambda t: [None], max_rows=0)):
            with pytest.raises(ValueError):
                bad()
        for bad in (lambda: eng.generate(p[0], 4, 0, 1, 0, sampling=dict(repetition=1.1)), lambda: eng.generate_tree(p, 4, lambda t: [None], sampling=dict(heat=1.0))):
            with pytest.raises(TypeError):
                bad()
        with pytest.raises(binding().LaError):
            eng.generate_tree(p, 40, lambda t: [None], n_pages=2)
        tokens, st = eng.generate_tree(p, 0, lambda t: [None])
        assert tokens.shape == (1, 0) and st["steps"] == 0 and st["free_pages"] == st["pages"]
    finally:
        eng.close()


# ---- captured, on streams ----------------------------------------------------------------------------------
class Step:
    """A batch's drafted step, all of it on the device, the drafts among it (the same tree for every request, tokens by a rule)."""
    PARENT = [-1, 0, 0, 1, 2, 3, 9, 5]

    def __init__(self, R=5, page=16, seed=0, layers=2):
        self.B, self.R, self.page, n = binding(), R, page, len(self.PARENT)
        self.shape, self.n = synth.SHAPES["small_bf16"].with_layers(layers), n
        self.eng = gpu_engine(self.shape, 64, seed=seed)
        self.k = torch.zeros((layers, 64, 2, page, 128), dtype=torch.bfloat16, device="cuda")
        self.pages = self.B.la_pages(self.k, torch.zeros_like(self.k))
        self.table, self.ring = torch.full((R, 40), -1, dtype=torch.int32, device="cuda"), torch.randperm(64, generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
        self.heads, self.heads_out, N = i32([0, 64, 0, 0]), i32([0] * 4), R * n
        self.len, self.grown, self.new_len = i32([0] * R), i32([0] * R), i32([0] * R)
        self.slot, self.pos, self.req, self.first, self.vis = i32([0] * N), i32([0] * N), i32([0] * N), i32([0] * (R + 1)), i64([0] * N)
        self.some = [i32([0]) for _ in range(3)] + [i32([0] * (R + 1))]
        self.parent, self.tok, self.ids = i32(self.PARENT * R), i32([0] * N), i32([0] * N)
        self.root = i32([7 * r + 3 for r in range(R)])
        self.hidden, self.logits, self.u = torch.zeros((N, 512), device="cuda"), torch.zeros((N, 2048), device="cuda"), torch.rand(400, generator=torch.Generator().manual_seed(9)).cuda()
        self.temperature, self.top_k = torch.full((N,), 0.5, device="cuda"), i32([3] * N)
        self.n_new, self.last = i32([0] * R), i32([0] * R)
        self.out, self.frm, self.to = (torch.full((R, 5), -1, dtype=torch.int32, device="cuda") for _ in range(3))
        self.tokens, self.n_tokens = torch.full((R, 400), -1, dtype=torch.int32, device="cuda"), i32([1] * R)
        self.tokens[:, 0] = self.root
        self.rep, self.allowed = torch.full((R,), 1.2, device="cuda"), torch.zeros((1, 64), dtype=torch.int32, device="cuda")
        self.allowed[0, 3] = 0b11110  # (four tokens, so that some drafts are right)
        self.which = i32([-1 if i % 11 == 10 else 0 for i in range(N)])

    def run(self):
        B, R, n = self.B, self.R, self.n
        self.tok.view(R, n).copy_((self.root[:, None] * 5 + torch.arange(n, device="cuda")[None] * 3) % 4 + 97)
        self.tok.view(R, n)[:, 0].copy_(self.root)
        torch.add(self.len, n, out=self.grown)
        B.la_page_map(self.len, self.grown, self.page, self.table, self.ring, self.heads, self.heads_out, self.slot, self.pos, self.req, self.first)
        B.la_tree_layout(self.parent, self.first, self.len, self.pos, self.vis)
        B.la_embed(self.eng.model, self.tok, self.hidden)
        B.la_forward_tree(self.eng.model, 0, self.shape.n_layers, self.hidden, self.pos, self.vis, self.slot, self.first, self.len, n, self.pages, self.table)
        B.la_unembed_logits(self.eng.model, self.hidden, self.logits)
        B.la_logits_adjust(self.logits, self.logits, req=self.req, repetition=self.rep, tokens=self.tokens, n_tokens=self.n_tokens, draft=self.tok, first=self.first, vis=self.vis,
                           allowed=self.allowed, allowed_index=self.which)
        B.la_sample(self.logits, self.u, self.ids, temperature=self.temperature, top_k=self.top_k, u_index=self.pos)
        B.la_tree_accept(self.parent, self.tok, self.ids, self.slot, self.first, self.len, self.n_new, self.new_len, self.last, self.out, self.frm, self.to)
        B.la_paged_copy(self.pages, self.frm, self.to)
        B.la_page_map(self.grown, self.new_len, self.page, self.table, self.ring, self.heads_out, self.heads, *self.some)
        at = torch.arange(5, device="cuda")[None]
        to = torch.where(at < self.n_new[:, None], self.n_tokens[:, None] + at, 399).long()
        self.tokens.scatter_(1, to, torch.where(at < self.n_new[:, None], self.out, -1))
        self.n_tokens.add_(self.n_new)
        self.len.copy_(self.new_len)
        self.root.copy_(self.out.gather(1, (self.n_new[:, None] - 1).clamp(min=0).long())[:, 0])

    def state(self):
        names = ("table", "ring", "heads", "slot", "pos", "req", "first", "vis", "tok", "ids", "hidden", "logits", "n_new", "new_len", "last", "out", "frm", "to", "tokens", "n_tokens", "root", "k")
        return [getattr(self, n).clone() for n in names] + [self.pages.v.clone()]


@pytest.mark.parametrize("first_captured", [False, True])
def test_a_captured_step_replays_as_the_eager_one(first_captured):
    """A drafted generation as one graph, replayed between other calls on the model, against the same steps made one by one; the model's first call may be the captured one."""
    eager, graphed = Step(), Step()
    try:
        if not first_captured:
            warm = Step()
            warm.run()
            graphed.B.la_forward_tree(graphed.eng.model, 0, 1, graphed.hidden.clone(), graphed.pos, graphed.vis, torch.full_like(graphed.slot, -1), graphed.first, graphed.len, 8, graphed.pages, graphed.table)
            warm.eng.close()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=torch.cuda.Stream()):
            graphed.run()
        accepted = 0
        for step in range(25):
            eager.run()
            g.replay()
            if step % 9 == 4:  # other calls on the same model and cache between the replays
                graphed.B.la_unembed_argmax(graphed.eng.model, graphed.hidden, i32([0] * 40))
                graphed.B.la_prefill(graphed.eng.model, graphed.eng.kv, i32(list(range(40))))
                torch.cuda.synchronize()
            for a, b in zip(eager.state(), graphed.state()):
                assert torch.equal(a, b), f"step {step}"
            accepted += int((eager.n_new > 1).sum())
        assert eager.heads.tolist()[3] == 0 and (eager.n_tokens == eager.len + 1).all() and accepted > 0
    finally:
        eager.eng.close()
        graphed.eng.close()


def attend_case(seed, R, ctx, rows, dtype=torch.bfloat16, page=16, heads=8):
    g, rng = torch.Generator(device="cuda").manual_seed(seed), random.Random(seed)
    blocks = (ctx + rows + page - 1) // page
    k, v = (torch.randn((1, R * blocks, 2, page, 128), generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.randperm(R * blocks, generator=g, device="cuda").to(torch.int32).view(R, blocks)
    q = torch.randn((R * rows, heads, 128), generator=g, device="cuda").to(dtype)
    vis = i64([m for _ in range(R) for _, m in paths(random_tree(rng, rows))])
    return binding().la_pages(k, v), q, table, i32([rows * r for r in range(R + 1)]), i32([rng.randint(0, ctx) for _ in range(R)]), vis


def adjust_case(seed, B, V):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.rand(s, generator=g, device="cuda")
    return torch.randn((B, V), generator=g, device="cuda"), dict(repetition=1 + r(B), presence=r(B), tokens=(r(B, 900) * V).to(torch.int32), n_tokens=i32([900] * B), bias=r(B, 30),
                                                                 bias_token=(r(B, 30) * V).to(torch.int32))


@pytest.mark.parametrize("rows,heads", [(3, 8), (20, 8), (64, 8)])
def test_calls_on_two_streams_at_once(rows, heads):
    """Each call has its own workspace: two streams' attention and adjustment, enqueued in turn, give what they give alone."""
    B = binding()
    cases, logits = [attend_case(s, 4, 3000, rows, heads=heads) for s in (1, 2)], [adjust_case(s, 4, 50000) for s in (3, 4)]

    def go(i, out, y, stream=None):
        pages, q, table, first, lens, vis = cases[i]
        B.la_paged_tree_attend(pages, 0, q, table, first, lens, vis, rows, out, stream=stream)
        B.la_logits_adjust(logits[i][0], y, stream=stream, **logits[i][1])

    want = []
    for i in range(2):
        out, y = torch.empty_like(cases[i][1]), torch.empty_like(logits[i][0])
        go(i, out, y)
        torch.cuda.synchronize()
        want.append((out, y))
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[(torch.zeros_like(cases[i][1]), torch.zeros_like(logits[i][0])) for _ in range(12)] for i in range(2)]
    torch.cuda.synchronize()
    for n in range(12):
        for i in range(2):
            go(i, *got[i][n], stream=streams[i])
            torch.empty(1 << 20, dtype=torch.uint8, device="cuda").fill_(255)  # (what the workspaces' memory might be given to)
    torch.cuda.synchronize()
    for i in range(2):
        for out, y in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(y, want[i][1])


def test_two_graphs_replayed_in_turn():
    B = binding()
    made = []
    for s in (5, 6):
        pages, q, table, first, lens, vis = attend_case(s, 3, 2500, 24)
        x, how = adjust_case(s, 2, 40000)
        out, y = torch.zeros_like(q), torch.zeros_like(x)

        def run(pages=pages, q=q, table=table, first=first, lens=lens, vis=vis, x=x, how=how, out=out, y=y):
            B.la_paged_tree_attend(pages, 0, q, table, first, lens, vis, 24, out)
            B.la_logits_adjust(x, y, **how)

        run()
        want = (out.clone(), y.clone())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        made.append((g, out, y, want, run))  # (run holds the tensors that the graph reads)
    for _ in range(4):
        for g, out, y, want, _run in made:
            out.zero_(), y.zero_()
            g.replay()
            junk = torch.full((1 << 22,), 3.0, device="cuda") * 2
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(y, want[1])
            del junk


@pytest.mark.parametrize("rows", [2, 64])
def test_lengths_and_rows_on_the_device_decide(rows):
    """A captured attention follows the lengths and the rows that stand in memory when it is replayed, from no key to all."""
    B = binding()
    pages, q, table, first, lens, vis = attend_case(11, 4, 4000, rows)
    out = torch.zeros_like(q)
    B.la_paged_tree_attend(pages, 0, q, table, first, lens, vis, rows, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.la_paged_tree_attend(pages, 0, q, table, first, lens, vis, rows, out)
    for ls, fs in (([0] * 4, None), ([4000] * 4, None), ([-1, 5, 3000, 17], [0, 1, 1, 2, 3]), ([1, 2, 3999, 0], [0, 0, 0, rows, rows]), ([511, 512, 513, 127], [1, 2, 3, 4, 4])):
        lens.copy_(i32(ls))
        first.copy_(i32(fs or [rows * r for r in range(5)]))
        out.fill_(5)
        g.replay()
        want = torch.zeros_like(q)
        B.la_paged_tree_attend(pages, 0, q, table, first, lens, vis, rows, want)
        assert torch.equal(out, want)


# ---- refusals of the binding --------------------------------------------------------------------------------
def test_binding_refuses_what_does_not_fit():
    B = binding()
    pages, q, table, first, lens, vis = attend_case(1, 3, 100, 4)
    out, n = torch.empty_like(q), i32([0] * 12)
    attend = lambda pages=pages, q=q, table=table, first=first, lens=lens, vis=vis, rows=4, out=out, layer=0: B.la_paged_tree_attend(pages, layer, q, table, first, lens, vis, rows, out)
    r, path, x = i32([0] * 3), torch.zeros((3, 4), dtype=torch.int32, device="cuda"), torch.zeros((3, 64), device="cuda")
    accept = lambda parent=n, tok=n, ids=n, slot=n, first=first, lens=lens, a=r, b=r, c=r, out=path, f=path, t=path, limit=None: B.la_tree_accept(parent, tok, ids, slot, first, lens, a, b, c, out, f, t, limit=limit)
    f3, t3 = torch.ones(3, device="cuda"), i32([[1, 2]] * 3)
    adjust = lambda x=x, y=x, **how: B.la_logits_adjust(x, y, **how)
    bad = [
        lambda: attend(q=q.float()), lambda: attend(out=out.float()), lambda: attend(vis=vis[:5]), lambda: attend(vis=vis.int()), lambda: attend(first=first[:3]), lambda: attend(first=first.long()),
        lambda: attend(lens=lens[:2]), lambda: attend(table=table.long()), lambda: attend(table=table[:2]), lambda: attend(rows=0), lambda: attend(rows=65), lambda: attend(layer=1), lambda: attend(q=q[:, :, :64]),
        lambda: attend(out=out[:1].expand(12, -1, -1)), lambda: attend(q=q.cpu()), lambda: attend(q=q[0]),
        lambda: B.la_tree_layout(n, first, lens, n[:5], vis), lambda: B.la_tree_layout(n, first, lens, n, n), lambda: B.la_tree_layout(n, first[:3], lens, n, vis), lambda: B.la_tree_layout(n.view(3, 4), first, lens, n, vis),
        lambda: B.la_tree_layout(n.long(), first, lens, n, vis), lambda: accept(tok=n[:5]), lambda: accept(ids=n.long()), lambda: accept(first=first[:2]), lambda: accept(a=n), lambda: accept(out=path[:2]),
        lambda: accept(f=path[:, :3]), lambda: accept(limit=n), lambda: accept(out=torch.zeros((3, 65), dtype=torch.int32, device="cuda"), f=torch.zeros((3, 65), dtype=torch.int32, device="cuda"), t=torch.zeros((3, 65), dtype=torch.int32, device="cuda")),
        lambda: accept(parent=n.view(3, 4)), lambda: accept(t=path.t().contiguous().t()),
        lambda: B.la_paged_copy(pages, n, n[:5]), lambda: B.la_paged_copy(pages, n.long(), n.long()), lambda: B.la_paged_copy(pages, n, n, run=65), lambda: B.la_paged_copy(pages, n, n, layers=(0, 2)),
        lambda: B.la_paged_copy(pages, n, n, run=0), lambda: B.la_paged_copy(pages, n[::2], n[::2]), lambda: B.la_paged_copy(pages, n.cpu(), n.cpu()),
        lambda: adjust(x=x.double(), y=x.double()), lambda: adjust(y=x[:2]), lambda: adjust(y=x.half()), lambda: adjust(x=x.t(), y=x.t()), lambda: adjust(repetition=f3[:2], n_requests=3), lambda: adjust(repetition=f3.half()),
        lambda: adjust(req=r[:2], repetition=f3), lambda: adjust(tokens=t3), lambda: adjust(tokens=t3, n_tokens=r[:2]), lambda: adjust(tokens=t3.long(), n_tokens=r), lambda: adjust(bias=t3.float()),
        lambda: adjust(bias=t3.float(), bias_token=t3[:, :1]), lambda: adjust(allowed=t3[:, :1]), lambda: adjust(allowed=t3[:1]), lambda: adjust(draft=r, vis=vis[:3]), lambda: adjust(draft=r, first=first, vis=vis),
        lambda: adjust(x=x[:1].expand(3, -1), y=x), lambda: adjust(repetition=f3[:2]), lambda: adjust(allowed=t3, allowed_index=r.long()), lambda: adjust(x=x.cpu(), y=x.cpu()),
    ]
    for i, call in enumerate(bad):
        with pytest.raises(B.LaError) as e:
            call()
        assert e.value.code in (-1, -3), i
    attend(), accept(), adjust(allowed=t3), adjust(repetition=f3, tokens=t3, n_tokens=r)  # (what the refused ones differ from)


def test_model_calls_refuse_what_does_not_fit(monkeypatch):
    B = binding()
    shape = synth.SHAPES["small_bf16"].with_layers(2)
    eng = gpu_engine(shape, 64)
    monkeypatch.setenv("LA_LDS_RING", "1")
    ring = gpu_engine(shape, 64)
    try:
        h, pages = torch.zeros((2, 512), device="cuda"), lambda L=2, dh=128, H=2, dt=torch.bfloat16: B.la_pages(*(torch.zeros((L, 4, H, 16, dh), dtype=dt, device="cuda") for _ in range(2)))
        two, table, vis, first, lens = i32([0, 1]), i32([[0, 1], [2, 3]]), i64([1, 1]), i32([0, 1, 2]), i32([0, 0])
        go = lambda h=h, pos=two, vis=vis, slot=two, first=first, lens=lens, rows=1, pages=pages(), table=table, lb=0, le=2, eng=eng: B.la_forward_tree(eng.model, lb, le, h, pos, vis, slot, first, lens, rows, pages, table)
        many = lambda n: dict(h=torch.zeros((n, 512), device="cuda"), pos=i32([0] * n), vis=i64([1] * n), slot=i32([0] * n))
        for n, (call, code) in enumerate([
                (lambda: go(h=torch.zeros((2, 256), device="cuda")), -1), (lambda: go(**many(65)), -1), (lambda: go(pages=pages(L=1)), -3), (lambda: go(pages=pages(dh=64)), -1), (lambda: go(pages=pages(H=4)), -1),
                (lambda: go(pages=pages(dt=torch.float16)), -1), (lambda: go(le=3), -3), (lambda: go(lb=2, le=1), -3), (lambda: go(lb=-1), -3), (lambda: go(rows=0), -1), (lambda: go(rows=65), -1),
                (lambda: go(pos=two[:1]), -1), (lambda: go(vis=vis.int()), -1), (lambda: go(first=first[:2]), -1), (lambda: go(lens=two[:1]), -1), (lambda: go(eng=ring), -1),
                (lambda: go(table=torch.zeros((65, 2), dtype=torch.int32, device="cuda"), first=i32([0] * 66), lens=i32([0] * 65)), -1)]):
            with pytest.raises(B.LaError) as e:
                call()
            assert e.value.code == code, n
        go()
    finally:
        eng.close()
        ring.close()
