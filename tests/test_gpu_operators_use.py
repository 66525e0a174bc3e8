"""The shared cache, sampling and stored logits as programs use them: captured and replayed, on several streams, refused; a step of all of them together."""
from types import SimpleNamespace

import pytest
import torch

import synth
from gpu_util import gpu_engine

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


def binding():
    from paper_2602_16760_amd import binding as B
    return B


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Step:
    """What a batch's step keeps: a model with a head, pages, tables, and the buffers of the calls."""

    def __init__(self, R=5, page=16, seed=0, layers=2):
        self.B, self.R, self.page = binding(), R, page
        self.shape = synth.SHAPES["small_bf16"].with_layers(layers)
        self.eng = gpu_engine(self.shape, 64, seed=seed)
        self.k = torch.zeros((layers, 64, 2, page, 128), dtype=BF16, device="cuda")
        self.pages = self.B.la_pages(self.k, torch.zeros_like(self.k))
        self.table, self.ring = torch.full((R, 40), -1, dtype=torch.int32, device="cuda"), torch.randperm(64, generator=torch.Generator().manual_seed(seed)).to(torch.int32).cuda()
        self.heads, self.heads_out = i32([0, 64, 0, 0]), i32([0] * 4)
        self.old, self.new = i32([0] * R), i32([1] * R)
        self.slot, self.pos, self.req, self.first = i32([0] * R), i32([0] * R), i32([0] * R), i32([0] * (R + 1))
        self.tok = i32([7 * r + 3 for r in range(R)])
        self.hidden = torch.zeros((R, 512), device="cuda")
        self.logits, self.u, self.ids, self.prob = torch.zeros((R, 2048), device="cuda"), torch.rand(R, generator=torch.Generator().manual_seed(9)).cuda(), i32([0] * R), torch.zeros(R, device="cuda")
        self.how = dict(temperature=torch.full((R,), 0.8, device="cuda"), top_k=i32([0, 5, 50, 1, 2048][:R]), top_p=torch.tensor([0.9, 1.0, 0.8, 1.0, 0.99][:R], device="cuda"))

    def run(self):
        """One token of every request, all of it on the device: pages, embedding, layers, logits, sample, and what the next step starts from."""
        B = self.B
        B.la_page_map(self.old, self.new, self.page, self.table, self.ring, self.heads, self.heads_out, self.slot, self.pos, self.req, self.first)
        B.la_embed(self.eng.model, self.tok, self.hidden)
        B.la_forward_paged(self.eng.model, 0, self.shape.n_layers, self.hidden, self.pos, self.req, self.slot, self.pages, self.table)
        B.la_unembed_logits(self.eng.model, self.hidden, self.logits)
        B.la_sample(self.logits, self.u, self.ids, self.prob, **self.how)
        self.heads.copy_(self.heads_out)
        self.old.copy_(self.new)
        self.new.add_(1)
        self.tok.copy_(self.ids)

    def state(self):
        return [t.clone() for t in (self.table, self.ring, self.heads, self.slot, self.pos, self.req, self.first, self.pages.k, self.pages.v, self.hidden, self.logits, self.ids, self.prob)]


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("first_captured", [False, True])
def test_a_captured_step_replays_as_the_eager_one(first_captured):
    """A generation of a batch as one graph, replayed between other calls on the model, against the same steps made one by one; the model's first call may be the captured one
    (its scratch memory is the model's)."""
    eager, graphed = Step(), Step()
    try:
        if not first_captured:
            warm = Step()
            warm.run()
            graphed.B.la_forward_paged(graphed.eng.model, 0, 1, graphed.hidden.clone(), graphed.pos, graphed.req, i32([-1] * 5), graphed.pages, graphed.table)
            warm.eng.close()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        side = torch.cuda.Stream()
        with torch.cuda.graph(g, stream=side):
            graphed.run()
        for step in range(40):
            eager.run()
            g.replay()
            if step % 9 == 4:  # other calls on the same model and cache between the replays
                graphed.B.la_unembed_argmax(graphed.eng.model, graphed.hidden, i32([0] * 5))
                graphed.B.la_prefill(graphed.eng.model, graphed.eng.kv, i32(list(range(40))))
                torch.cuda.synchronize()
            assert same(eager.state(), graphed.state()), f"step {step}"
        assert eager.heads.tolist() == [15, 49, 5, 0] and eager.pos.tolist() == [39] * 5
    finally:
        eager.eng.close()
        graphed.eng.close()


def attend_case(seed, rows, ctx, dtype=BF16, page=16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    blocks = (ctx + page - 1) // page
    k, v = (torch.randn((1, rows * blocks, 2, page, 128), generator=g, device="cuda").to(dtype) for _ in range(2))
    table = torch.randperm(rows * blocks, generator=g, device="cuda").to(torch.int32).view(rows, blocks)
    q = torch.randn((rows, 8, 128), generator=g, device="cuda").to(dtype)
    pos = torch.randint(0, ctx, (rows,), generator=g, device="cuda").to(torch.int32)
    return binding().la_pages(k, v), q, table, pos


def test_calls_on_two_streams_at_once():
    """Each call has its own workspace: two streams' attention and sampling, enqueued in turn, give what they give alone."""
    B = binding()
    cases = [attend_case(s, 6, 3000) for s in (1, 2)]
    rows = [torch.randn((4, 50000), generator=torch.Generator(device="cuda").manual_seed(s), device="cuda") for s in (3, 4)]
    u, p = torch.tensor([0.1, 0.5, 0.7, 0.999], device="cuda"), torch.tensor([0.9, 1.0, 0.5, 0.99], device="cuda")

    def go(i, out, ids, stream=None):
        pages, q, table, pos = cases[i]
        B.la_paged_attend(pages, 0, q, table, None, pos, out, stream=stream)
        B.la_sample(rows[i], u, ids, top_p=p, stream=stream)

    want = []
    for i in range(2):
        out, ids = torch.empty_like(cases[i][1]), i32([0] * 4)
        go(i, out, ids)
        torch.cuda.synchronize()
        want.append((out, ids))
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [[(torch.zeros_like(cases[i][1]), i32([0] * 4)) for _ in range(20)] for i in range(2)]
    torch.cuda.synchronize()
    for n in range(20):
        for i in range(2):
            go(i, *got[i][n], stream=streams[i])
            torch.empty(1 << 20, dtype=torch.uint8, device="cuda").fill_(255)  # (what the workspaces' memory might be given to)
    torch.cuda.synchronize()
    for i in range(2):
        for out, ids in got[i]:
            assert torch.equal(out, want[i][0]) and torch.equal(ids, want[i][1])


def test_two_graphs_replayed_in_turn():
    B = binding()
    made = []
    for s in (5, 6):
        pages, q, table, pos = attend_case(s, 3, 2500)
        x, u, out, ids = torch.randn((2, 40000), device="cuda"), torch.rand(2, device="cuda"), torch.zeros_like(q), i32([0, 0])

        def run(pages=pages, q=q, table=table, pos=pos, x=x, u=u, out=out, ids=ids):
            B.la_paged_attend(pages, 0, q, table, None, pos, out)
            B.la_sample(x, u, ids, min_p=torch.full((2,), 0.01, device="cuda"))

        run()
        want = (out.clone(), ids.clone())
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            run()
        made.append((g, out, ids, want, run))  # (run holds the tensors that the graph reads)
    for _ in range(4):
        for g, out, ids, want, _run in made:
            out.zero_(), ids.fill_(-7)
            g.replay()
            junk = torch.full((1 << 22,), 3.0, device="cuda") * 2
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(ids, want[1])
            del junk


def test_lengths_on_the_device_decide():
    """A captured attention follows the positions that stand in memory when it is replayed, from one key to all."""
    B = binding()
    pages, q, table, pos = attend_case(11, 4, 4000)
    out = torch.zeros_like(q)
    B.la_paged_attend(pages, 0, q, table, None, pos, out)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.la_paged_attend(pages, 0, q, table, None, pos, out)
    for lens in ([0, 0, 0, 0], [3999] * 4, [-1, 5, 3000, 17], [1, -1, -1, 3999], [511, 512, 513, 127]):
        pos.copy_(i32(lens))
        g.replay()
        want = torch.zeros_like(q)
        B.la_paged_attend(pages, 0, q, table, None, pos, want)
        assert torch.equal(out, want)


# ---- refusals of the binding --------------------------------------------------------------------------------
def test_binding_refuses_what_does_not_fit():
    B = binding()
    from paper_2602_16760_amd.binding import LaError
    pages, q, table, pos = attend_case(1, 3, 100)
    out, f, x = torch.empty_like(q), torch.zeros(3, device="cuda"), torch.zeros((3, 64), device="cuda")
    ids, k = i32([0] * 3), torch.zeros((3, 2, 128), dtype=BF16, device="cuda")
    first = i32([0] * 4)
    four, ring = i32([0] * 4), i32(list(range(9)))
    bad = [
        lambda: B.la_paged_attend(pages, 0, q.float(), table, None, pos, out), lambda: B.la_paged_attend(pages, 0, q, table, None, pos, out.float()),
        lambda: B.la_paged_attend(pages, 0, q, table, None, pos[:2], out), lambda: B.la_paged_attend(pages, 0, q, table.long(), None, pos, out),
        lambda: B.la_paged_attend(pages, 0, q, table, pos[:1], pos, out), lambda: B.la_paged_attend(pages, 0, q[:, :, :64], table, None, pos, out[:, :, :64]),
        lambda: B.la_paged_attend(pages, 0, q, table.t().contiguous().t(), None, pos, out), lambda: B.la_paged_attend(pages, 0, q[:, ::2], table, None, pos, out[:, ::2]),
        lambda: B.la_paged_attend(pages, 1, q, table, None, pos, out), lambda: B.la_paged_attend(pages, 0, q, table[:2], None, pos, out),
        lambda: B.la_paged_attend(pages, 0, q, table, None, pos, out[:1].expand(3, -1, -1)), lambda: B.la_paged_attend(pages, 0, q.cpu(), table, None, pos, out),
        lambda: B.la_paged_write(pages, 0, k, k[:2], ids), lambda: B.la_paged_write(pages, 0, k, k, ids[:2]), lambda: B.la_paged_write(pages, 0, k, k.float(), ids),
        lambda: B.la_paged_write(pages, 5, k, k, ids), lambda: B.la_pages(pages.k, pages.v[:, :4]), lambda: B.la_pages(pages.k, pages.v.float()), lambda: B.la_pages(pages.k[0], pages.v[0]),
        lambda: B.la_sample(x.double(), f, ids), lambda: B.la_sample(x, f[:2], ids), lambda: B.la_sample(x, f, ids[:2]), lambda: B.la_sample(x, f, ids.long()),
        lambda: B.la_sample(x, f, ids, temperature=ids), lambda: B.la_sample(x, f, ids, top_k=f), lambda: B.la_sample(x.t(), f, ids), lambda: B.la_sample(x, f, ids, prob=f[:1]),
        lambda: B.la_sample(x, f.cpu(), ids), lambda: B.la_sample(x[0], f, ids), lambda: B.la_sample(x[:1].expand(3, -1), f, ids),
        lambda: B.la_page_map(ids, ids, 16, table, ring, four, four, ids, ids, ids, first), lambda: B.la_page_map(ids, ids[:2], 16, table, ring, four, i32([0] * 4), ids, ids, ids, first),
        lambda: B.la_page_map(ids, ids, 0, table, ring, four, i32([0] * 4), ids, ids, ids, first), lambda: B.la_page_map(ids, ids, 16, table, ring, four, i32([0] * 4), ids, ids, ids, ids),
        lambda: B.la_page_map(ids, ids, 16, table, ring, four, i32([0] * 4), ids, ids[:2], ids, first),
    ]
    for n, call in enumerate(bad):
        with pytest.raises(LaError) as e:
            call()
        assert e.value.code in (-1, -3), n


def test_model_calls_refuse_what_does_not_fit():
    B = binding()
    shape = synth.SHAPES["small_bf16"].with_layers(2)
    eng, headless = gpu_engine(shape, 64), gpu_engine(shape, 64, head=False)
    try:
        h, pages = torch.zeros((2, 512), device="cuda"), lambda L=2, dh=128, H=2, dt=BF16: B.la_pages(*(torch.zeros((L, 4, H, 16, dh), dtype=dt, device="cuda") for _ in range(2)))
        two, table = i32([0, 1]), i32([[0, 1], [2, 3]])
        go = lambda h=h, pos=two, req=two, slot=two, pages=pages(), table=table, lb=0, le=2: B.la_forward_paged(eng.model, lb, le, h, pos, req, slot, pages, table)
        for n, (call, code) in enumerate([
                (lambda: B.la_unembed_logits(eng.model, h, torch.zeros((2, 2047), device="cuda")), -1), (lambda: B.la_unembed_logits(eng.model, h, torch.zeros((3, 2048), device="cuda")), -1),
                (lambda: B.la_unembed_logits(eng.model, h[:, :256], torch.zeros((2, 2048), device="cuda")), -1), (lambda: B.la_unembed_logits(headless.model, h, torch.zeros((2, 2048), device="cuda")), -1),
                (lambda: B.la_unembed_logits(eng.model, torch.zeros((65, 512), device="cuda"), torch.zeros((65, 2048), device="cuda")), -1),
                (lambda: go(h=torch.zeros((2, 256), device="cuda")), -1), (lambda: go(h=torch.zeros((65, 512), device="cuda"), pos=i32([0] * 65), req=i32([0] * 65), slot=i32([0] * 65)), -1),
                (lambda: go(pages=pages(L=1)), -3), (lambda: go(pages=pages(dh=64)), -1), (lambda: go(pages=pages(H=4)), -1), (lambda: go(pages=pages(dt=torch.float16)), -1), (lambda: go(le=3), -3),
                (lambda: go(lb=2, le=1), -3), (lambda: go(lb=-1), -3), (lambda: go(req=None, table=table[:1]), -1), (lambda: go(pos=two[:1]), -1)]):
            with pytest.raises(B.LaError) as e:
                call()
            assert e.value.code == code, n
    finally:
        eng.close()
        headless.close()


def test_the_other_weight_layout_is_refused(monkeypatch):
    monkeypatch.setenv("LA_LDS_RING", "1")
    B = binding()
    shape = synth.SHAPES["small_bf16"].with_layers(1)
    eng = gpu_engine(shape, 64)
    try:
        with pytest.raises(B.LaError):
            B.la_unembed_logits(eng.model, torch.zeros((1, 512), device="cuda"), torch.zeros((1, 2048), device="cuda"))
        with pytest.raises(B.LaError):
            B.la_forward_paged(eng.model, 0, 1, torch.zeros((1, 512), device="cuda"), i32([0]), None, i32([0]), B.la_pages(*(torch.zeros((1, 1, 2, 16, 128), dtype=BF16, device="cuda") for _ in range(2))),
                               i32([[0]]))
    finally:
        eng.close()


@pytest.mark.parametrize("wgs", ["37", "256"])
def test_logits_of_other_stream_counts_and_the_greedy_head_agree(wgs, monkeypatch):
    """The largest stored logit is the arg-max's wherever the two best are further apart than the arg-max's operand rounds (2^-11 of the row's size), at any packing of the head."""
    monkeypatch.setenv("LA_WGS", wgs)
    B = binding()
    g = torch.Generator().manual_seed(4)
    d, V = 512, 5008
    gain, un = torch.rand(d, generator=g) + 0.5, (torch.randn((d, V), generator=g) * 0.02).to(BF16)
    model = B.la_init_model(SimpleNamespace(n_layers=1, d_model=d, n_q_heads=1, n_kv_heads=1, head_dim=64, d_ffn=64, vocab=V, rms_eps=1e-5, rope_theta=1e4, dtype="bf16"), None, gain.cuda(), un.cuda())
    torch.cuda.synchronize()
    try:
        h = torch.randn((64, d), generator=g).cuda()
        logits, ids, top2 = torch.empty((64, V), device="cuda"), i32([0] * 64), torch.empty((64, 2), device="cuda")
        B.la_unembed_logits(model, h, logits)
        B.la_unembed_argmax(model, h, ids, top2)
        n = h.double().cpu()
        n = n * torch.rsqrt((n * n).mean(1, keepdim=True) + 1e-5) * gain.double()
        size = (n.abs() @ un.double().abs()).amax(1)
        best = logits.cpu().double().topk(2, dim=1)
        clear = (best.values[:, 0] - best.values[:, 1]) > 2.0 ** -10 * size
        assert torch.equal(best.indices[clear, 0].to(torch.int32), ids.cpu()[clear]) and (best.values[:, 0] - top2.cpu()[:, 0].double()).abs().le(2.0 ** -10 * size).all()
        zero = torch.zeros(64, device="cuda")
        picked = i32([0] * 64)
        B.la_sample(logits, zero, picked, temperature=zero)
        assert torch.equal(picked.cpu(), best.indices[:, 0].to(torch.int32))
    finally:
        B.la_free_model(model)
