"""Several requests at once: rows of them through the layers on pages, generation with shared pages, sampled generation."""
from dataclasses import replace

import numpy as np
import pytest
import torch

import synth
from gpu_util import gpu_engine, launch_names, oracle_model, row_rel_err
from oracle import transformer as otf

pytestmark = pytest.mark.gpu
BAR = {"f32": 1e-4, "bf16": 2e-2, "f16": 2e-3}


def binding():
    from paper_2602_16760_amd import binding as B
    return B


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def bits(a, dtype):
    """numpy rows of synth -> torch rows of the pages' type."""
    t = torch.from_numpy(np.ascontiguousarray(a))
    return t.view(torch.bfloat16) if dtype == "bf16" and t.dtype != torch.float32 else t.to(dict(f32=torch.float32, bf16=torch.bfloat16, f16=torch.float16)[dtype])


@pytest.mark.parametrize("name,lens,page,env", [("tiny_f32", [0, 5, 47, 300], 16, {}), ("small_bf16", [0, 1, 31, 33, 700], 16, {}), ("small_bf16", list(range(3, 67)), 24, {}),
                                                ("small64_bf16", [100, 2], 8, {}), ("small_f16", [64, 12, 1000], 32, {}), ("small64_f16", [7] * 17, 16, {}),
                                                ("small_bf16", [0, 40, 600], 16, {"LA_FORCE_GENERIC": "1"}), ("small64_f16", [5, 90, 1], 12, {"LA_FORCE_GENERIC": "1"}),
                                                ("small_bf16", [3, 33], 16, {"LA_WGS": "37"})])
def test_forward_against_the_oracle(name, lens, page, env, monkeypatch):
    """A row per request, one of the batch padding: hidden states against the oracle's decode step of each request, K and V where the slots say.  16-bit models also
    on the plain kernels, and with weights laid out for another number of workgroups."""
    for key, value in env.items():
        monkeypatch.setenv(key, value)
    shape = synth.SHAPES[name]
    eng, om, B = gpu_engine(shape, 64, head=False), oracle_model(shape, head=False), binding()
    R, H, dh, dt = len(lens), shape.n_kv_heads, shape.head_dim, shape.dtype
    try:
        blocks = max(lens) // page + 1
        n_pages = sum(n // page + 1 for n in lens)
        order = np.random.default_rng(2).permutation(n_pages)
        table = np.full((R, blocks), -1, dtype=np.int32)
        k = torch.zeros((shape.n_layers, n_pages, H, page, dh), dtype=bits(np.zeros(1, np.float32), dt).dtype)
        v, at, rows = torch.zeros_like(k), 0, []
        for r, n in enumerate(lens):
            u = n // page + 1
            table[r, :u] = order[at:at + u]
            at += u
            okv = otf.KVCache(shape, n + 1)
            for l in range(shape.n_layers):
                if n:
                    kk, vv = synth.kv_fill(shape, l, n, r)
                    okv.fill(l, kk, vv)
                    for dst, src in ((k, bits(kk, dt)), (v, bits(vv, dt))):
                        for b in range(u):
                            part = src[b * page:(b + 1) * page]
                            dst[l, table[r, b], :, :len(part)] = part.transpose(0, 1)
            okv.L = n
            rows.append(okv)
        x = synth.hidden_block(shape, R, 0)
        pad = min(3, R)
        B_rows = min(R + 1, 64)
        req, pos = list(range(R)), list(lens)
        slot = [int(table[r, n // page]) * page + n % page for r, n in enumerate(lens)]
        if B_rows > R:
            req.insert(pad, -1), pos.insert(pad, -1), slot.insert(pad, -1)
            x = np.insert(x, pad, 1.0, axis=0)
        pages = B.la_pages(k.cuda(), v.cuda())
        before = pages.k.clone()
        hidden = torch.from_numpy(x.astype(np.float32)).cuda()
        run = lambda h: B.la_forward_paged(eng.model, 0, shape.n_layers, h, i32(pos), i32(req), i32(slot), pages, i32(table.tolist()))
        used = launch_names(lambda: run(hidden.clone()))
        assert {"paged_attend"} <= used and ("pf_gemm_qkv" in used) == (dt != "f32" and "LA_FORCE_GENERIC" not in env), used
        run(hidden)
        got = hidden.cpu().numpy()
        again = torch.from_numpy(x.astype(np.float32)).cuda()
        run(again)
        assert torch.equal(again, hidden)
        touched = torch.zeros(pages.k.shape[1:4], dtype=torch.bool)
        for i, r in enumerate(req):
            if r < 0:
                continue
            want = otf.forward_block(om, rows[r], x[i:i + 1], [lens[r]], [1])
            err = row_rel_err(got[i:i + 1], want).max()
            assert err <= BAR[dt], f"request {r} of {lens[r]} positions: {err:.2e}"
            p, c = slot[i] // page, slot[i] % page
            touched[p, :, c] = True
            for cache, theirs in ((pages.k, rows[r].K), (pages.v, rows[r].V)):
                row = cache[shape.n_layers - 1, p, :, c].float().cpu().numpy()
                ref = np.asarray(theirs[shape.n_layers - 1][lens[r]], dtype=np.float64).reshape(H, dh)
                assert np.abs(row - ref).max() <= (BAR[dt] + 2.0 ** -8) * np.abs(ref).max()
        assert torch.equal(pages.k.cpu()[:, ~touched], before.cpu()[:, ~touched])
    finally:
        eng.close()


@pytest.mark.parametrize("rows", [1, 16, 17, 40, 64])
@pytest.mark.parametrize("Hq,Hkv", [(8, 2), (64, 8)])
def test_forward_of_narrow_and_wide_qkv(Hq, Hkv, rows):
    """QKV products of one round of workgroups, and of more, at every number of row tiles: each row as it comes out alone, and against the oracle."""
    shape = replace(synth.SHAPES["small_bf16"], n_q_heads=Hq, n_kv_heads=Hkv, n_layers=1)
    eng, om, B = gpu_engine(shape, 64, head=False), oracle_model(shape, head=False), binding()
    try:
        pages = lambda: B.la_pages(*(torch.zeros((1, 70, Hkv, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        table = torch.randperm(70, generator=torch.Generator().manual_seed(rows))[:rows].to(torch.int32).cuda().view(rows, 1)
        slot, pos = (table[:, 0] * 16).contiguous(), i32([0] * rows)
        x = synth.hidden_block(shape, rows, 0)
        hidden, pg = torch.from_numpy(x.astype(np.float32)).cuda(), pages()
        B.la_forward_paged(eng.model, 0, 1, hidden, pos, None, slot, pg, table)
        for r in range(0, rows, 7):
            want = otf.forward_block(om, otf.KVCache(shape, 1), x[r:r + 1], [0], [1])
            assert row_rel_err(hidden[r:r + 1].cpu().numpy(), want).max() <= BAR["bf16"]
        alone, other = torch.from_numpy(x[-1:].astype(np.float32)).cuda(), pages()
        B.la_forward_paged(eng.model, 0, 1, alone, pos[:1], None, slot[-1:].contiguous(), other, table[-1:].contiguous())
        at = int(table[-1, 0])
        assert torch.equal(other.k[0, at], pg.k[0, at]) and torch.equal(other.v[0, at], pg.v[0, at])
    finally:
        eng.close()


def test_forward_in_ranges_of_layers_and_without_a_row_map():
    shape = synth.SHAPES["small_bf16"]
    eng, B = gpu_engine(shape, 64, head=False), binding()
    try:
        mk = lambda: B.la_pages(*(torch.zeros((3, 6, 2, 16, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2)))
        table, pos, slot = i32([[4, 2], [1, 0], [3, 5]]), i32([0, 0, 0]), i32([64, 16, 48])
        x = torch.from_numpy(synth.hidden_block(shape, 3, 1).astype(np.float32)).cuda()
        a, b, pa, pb = x.clone(), x.clone(), mk(), mk()
        B.la_forward_paged(eng.model, 0, 3, a, pos, i32([0, 1, 2]), slot, pa, table)
        for l in range(3):
            B.la_forward_paged(eng.model, l, l + 1, b, pos, None, slot, pb, table)
        assert torch.equal(pa.k, pb.k) and torch.equal(pa.v, pb.v) and torch.equal(a, b)
        B.la_forward_paged(eng.model, 1, 1, b, pos, None, slot, pb, table)
        assert torch.equal(a, b)
    finally:
        eng.close()


def greedy_is_the_oracles(shape, om, prompt, tokens, bar):
    """Every emitted token is the oracle's choice behind the tokens in front of it, wherever its margin is clear of the bar."""
    seq = np.concatenate([prompt, tokens]).astype(np.int64)
    logits = otf.causal_forward(om, seq[:-1])[1][len(prompt) - 1:]
    t1, t2 = otf.top2_margin(logits)
    safe = (t1 - t2) > bar
    assert np.array_equal(otf.argmax_ids(logits)[safe], tokens[safe])
    return int(safe.sum())


@pytest.mark.parametrize("name,margin", [("tiny_f32", 1e-3), ("small_bf16", 3e-2), ("small64_f16", 1e-2)])
def test_batch_generation_against_the_oracle(name, margin):
    shape = synth.SHAPES[name]
    eng, om = gpu_engine(shape, 300, seed=1), oracle_model(shape, seed=1)
    g = np.random.default_rng(5)
    prompts = [g.integers(0, shape.vocab, size=n).astype(np.int32) for n in (1, 9, 16, 17, 90, 150)]
    try:
        tokens, st = eng.generate_batch(prompts, 20, page_size=16)
        assert st["free_pages"] == st["pages"]
        safe = sum(greedy_is_the_oracles(shape, om, p, t, margin) for p, t in zip(prompts, tokens))
        assert safe >= 40, f"only {safe} of 120 tokens have a margin"
        with pytest.raises(Exception) as e:
            eng.generate_batch(prompts, 20, page_size=16, n_pages=st["pages"] - 1)
        assert getattr(e.value, "code", None) == -3
    finally:
        eng.close()


def test_batch_equals_each_request_alone_in_float32():
    """The tiny decoder's rounding is far below its margins: the batch emits what sequential decoding emits, greedily and sampled."""
    shape = synth.SHAPES["tiny_f32"]
    eng = gpu_engine(shape, 200, seed=2)
    g = np.random.default_rng(6)
    prompts = [g.integers(0, shape.vocab, size=n).astype(np.int32) for n in (5, 40, 23)]
    try:
        tokens, _ = eng.generate_batch(prompts, 24, page_size=8)
        for p, t in zip(prompts, tokens):
            assert np.array_equal(eng.generate(p, 24, 0, 1, 0)[0], t)
        u = g.random((24, 3)).astype(np.float32)
        how = dict(temperature=0.8, top_k=30, top_p=0.9, min_p=0.02)
        tokens, _ = eng.generate_batch(prompts, 24, page_size=8, sampling=dict(how, u=u))
        for r, p in enumerate(prompts):
            by_pos = np.zeros(200 + 1, dtype=np.float32)
            by_pos[len(p) - 1:len(p) - 1 + 24] = u[:, r]
            assert np.array_equal(eng.generate(p, 24, 0, 1, 0, sampling=dict(how, u=by_pos))[0], tokens[r])
    finally:
        eng.close()


@pytest.mark.parametrize("name,W,N,G", [("tiny_f32", 4, 3, 4), ("tiny_f32", 5, 4, 5), ("tiny_f32", 1, 2, 1)])
@pytest.mark.parametrize("how", [dict(temperature=0.7, top_k=8), dict(temperature=0.3, top_p=0.8), dict(temperature=0.0)])
def test_sampled_lookahead_emits_what_sequential_sampling_emits(name, W, N, G, how):
    """Random numbers go by position, so a candidate that its row draws is the token that sequential decoding would have drawn there; a low temperature confirms candidates."""
    shape = synth.SHAPES[name]
    eng = gpu_engine(shape, 400, seed=3)
    prompt = np.tile(np.random.default_rng(7).integers(0, shape.vocab, size=12), 4).astype(np.int32)
    try:
        one, _ = eng.generate(prompt, 60, 0, 1, 0, sampling=dict(how, seed=11))
        many, st = eng.generate(prompt, 60, W, N, G, sampling=dict(how, seed=11))
        assert np.array_equal(one, many)
        if how == dict(temperature=0.0):
            assert np.array_equal(one, eng.generate(prompt, 60, W, N, G)[0])
    finally:
        eng.close()


def test_sampling_parameters_are_checked():
    eng = gpu_engine(synth.SHAPES["tiny_f32"], 64)
    try:
        with pytest.raises(TypeError):
            eng.generate(np.array([1, 2, 3]), 4, 0, 1, 0, sampling=dict(heat=1.0))
        with pytest.raises(ValueError):
            eng.generate(np.array([1, 2, 3]), 4, 0, 1, 0, sampling=dict(u=[0.5]))
        with pytest.raises(ValueError):
            eng.generate_batch([], 4)
    finally:
        eng.close()


@pytest.mark.parametrize("lens,n_new", [([1], 0), ([4, 1], 0), ([1, 1, 1], 1), ([17], 1)])
def test_batches_of_next_to_nothing(lens, n_new):
    """Prompts of one token, no token or one to generate: the shapes, and the pages all given back."""
    shape = synth.SHAPES["small_bf16"]
    eng = gpu_engine(shape, 64)
    try:
        prompts = [np.arange(3, 3 + n) for n in lens]
        tokens, stats = eng.generate_batch(prompts, n_new)
        assert tokens.shape == (len(lens), n_new) and stats["free_pages"] == stats["pages"]
        for p, t in zip(prompts, tokens):
            alone, _ = eng.generate_batch([p], n_new)
            assert (alone[0] == t).all()
        with pytest.raises(binding().LaError):  # longer than the contiguous cache that prompts go through
            eng.generate_batch([np.zeros(100, dtype=np.int64)], 2)
    finally:
        eng.close()


@pytest.mark.parametrize("W,N,G", [(4, 3, 4), (5, 4, 5)])
@pytest.mark.parametrize("how", [dict(temperature=0.0), dict(temperature=0.05, top_p=0.95), dict(temperature=0.1, top_k=8), dict(temperature=1.5, top_k=2)])
def test_sampled_lookahead_confirms_candidates(W, N, G, how):
    """Behind a prompt that repeats itself candidates are what their rows draw: there are fewer steps than tokens, and the same tokens."""
    eng = gpu_engine(synth.SHAPES["tiny_f32"], 400, seed=3)
    prompt = np.tile(np.random.default_rng(7).integers(0, eng.shape.vocab, size=12), 4).astype(np.int32)
    try:
        one, alone = eng.generate(prompt, 60, 0, 1, 0, sampling=dict(how, seed=11))
        many, st = eng.generate(prompt, 60, W, N, G, sampling=dict(how, seed=11))
        assert np.array_equal(one, many)
        assert alone["steps"] == 60 and alone["matched_steps"] == 0 and 0 < st["matched_steps"] <= st["steps"] < 50
    finally:
        eng.close()


@pytest.mark.parametrize("name,margin", [("small_bf16", 3e-2), ("small64_f16", 1e-2)])
@pytest.mark.parametrize("temperature", [0.3, 0.7])
def test_sampled_tokens_of_16_bit_models_are_where_their_numbers_fall(name, margin, temperature):
    """Every token, of sequential and of lookahead decoding: in the oracle's distribution behind the tokens in front of it, the random number of its position falls into the token's
    share or next to it.  Logits within `margin` of the oracle's move a sum of shares by exp(2 margin / temperature) - 1 at most.  (A row's last bits go by the block that it
    stands in, so the two may part where a number falls on a border.)"""
    shape = synth.SHAPES[name]
    eng, om = gpu_engine(shape, 400, seed=3), oracle_model(shape, seed=3)
    W, N, G, matched = 4, 3, 4, 0
    delta = np.exp(2 * margin / temperature) - 1
    try:
        for seed in (7, 8):
            g = np.random.default_rng(seed)
            prompt, u = np.tile(g.integers(0, shape.vocab, size=12), 4).astype(np.int32), g.random(400 + 64).astype(np.float32)
            for which in ((0, 1, 0), (W, N, G)):
                tokens, st = eng.generate(prompt, 60, *which, sampling=dict(temperature=temperature, u=u))
                seq = np.concatenate([prompt, tokens]).astype(np.int64)
                x = otf.causal_forward(om, seq[:-1])[1][len(prompt) - 1:].astype(np.float64) / temperature
                w = np.exp(x - x.max(1, keepdims=True))
                ends = np.cumsum(w, 1) / w.sum(1, keepdims=True)
                i, at = np.arange(60), u[len(prompt) - 1:len(prompt) + 59]
                hi, lo = ends[i, tokens], ends[i, tokens] - (w / w.sum(1, keepdims=True))[i, tokens]
                assert ((at >= lo - delta) & (at <= hi + delta)).all()
                matched += st["matched_steps"]
        assert temperature > 0.5 or matched > 0
    finally:
        eng.close()


@pytest.mark.parametrize("n_pages,fits", [(8, False), (9, True)])
def test_a_batch_that_its_pages_do_not_hold_is_refused_before_its_prompts_run(n_pages, fits, monkeypatch):
    """1 + 60 and 20 + 60 positions of 16 a page: four and five pages at the last step, three with the prompts in."""
    shape = synth.SHAPES["tiny_f32"]
    eng, ran = gpu_engine(shape, 64), []
    prefill = eng.prefill
    monkeypatch.setattr(eng, "prefill", lambda *a, **k: (ran.append(1), prefill(*a, **k))[1])
    prompts = [np.arange(2), np.arange(21)]  # (the last token of a prompt is the first step's)
    try:
        if fits:
            tokens, st = eng.generate_batch(prompts, 60, n_pages=n_pages)
            assert tokens.shape == (2, 60) and st["free_pages"] == st["pages"] == n_pages and len(ran) == 2
        else:
            with pytest.raises(binding().LaError) as e:
                eng.generate_batch(prompts, 60, n_pages=n_pages)
            assert e.value.code == -3 and not ran
    finally:
        eng.close()


@pytest.mark.parametrize("name,page,env", [("tiny_f32", 8, {}), ("small_bf16", 16, {}), ("small64_f16", 12, {}), ("small_bf16", 16, {"LA_FORCE_GENERIC": "1"})])
def test_rows_of_one_request_see_each_other_up_to_their_own_positions(name, page, env, monkeypatch):
    """Two prompts in one call, rows in any order, and a second call behind them: a causal block of the oracle each."""
    for key, value in env.items():
        monkeypatch.setenv(key, value)
    shape = synth.SHAPES[name]
    eng, om, B = gpu_engine(shape, 64, head=False), oracle_model(shape, head=False), binding()
    try:
        dt = bits(np.zeros(1, np.float32), shape.dtype).dtype
        pages = B.la_pages(*(torch.full((shape.n_layers, 10, shape.n_kv_heads, page, shape.head_dim), float("nan"), dtype=dt, device="cuda") for _ in range(2)))
        table = i32([[7, 2, 9, 0, 4], [1, 8, 5, 3, 6]])
        okv, g = [otf.KVCache(shape, 40) for _ in range(2)], np.random.default_rng(4)
        done = [0, 0]
        for call, counts in enumerate([(24, 13), (6, 1), (1, 20)]):
            rows = [(r, done[r] + i) for r in range(2) for i in range(counts[r])]
            order = g.permutation(len(rows))
            x = synth.hidden_block(shape, len(rows), call)
            req, pos = [rows[i][0] for i in order], [rows[i][1] for i in order]
            slot = [int(table[r, p // page]) * page + p % page for r, p in zip(req, pos)]
            hidden = torch.from_numpy(x[order].astype(np.float32)).cuda()
            B.la_forward_paged(eng.model, 0, shape.n_layers, hidden, i32(pos), i32(req), i32(slot), pages, table)
            got = np.empty_like(x)
            got[order] = hidden.cpu().numpy()
            for r in range(2):
                mine = [i for i, row in enumerate(rows) if row[0] == r]
                okv[r].L = done[r]
                want = otf.forward_block(om, okv[r], x[mine], [rows[i][1] for i in mine], [(1 << (j + 1)) - 1 for j in range(len(mine))])
                assert row_rel_err(got[mine], want).max() <= BAR[shape.dtype], f"call {call}, request {r}"
                done[r] += counts[r]
    finally:
        eng.close()
