"""Host-side orchestration of the C-ABI calls: model upload, prefill, decode loops.

No arithmetic of the method lives here: every step (embedding gather, layer stack,
unembedding + argmax, n-gram acceptance, KV commit, next-block build) is a library call.
"""
from __future__ import annotations

import time

import numpy as np
import torch

from . import binding as B


class Engine:
    """One model + one KV cache + (optionally) one lookahead controller on cuda:0."""

    def __init__(self, shape, max_len: int, layer_source=None, head: dict | None = None):
        self.shape = shape
        self.max_len = max_len
        head = head or {}
        dev = {k: B.to_device(v) for k, v in head.items()}
        self.model = B.la_init_model(shape, dev.get("embed"), dev.get("g_final"), dev.get("unembed"))
        torch.cuda.synchronize()
        del dev
        if layer_source is not None:
            for l in range(shape.n_layers):
                self.set_layer(l, layer_source(l))
        self.kv = B.la_kv_alloc(self.model, max_len)
        self.pool = None
        self.state = None
        self.la = None
        self._sample = None

    def set_layer(self, l: int, w: dict):
        dev = {k: B.to_device(v) for k, v in w.items()}
        B.la_model_set_layer(self.model, l, dev)
        torch.cuda.synchronize()  # the library has packed its own copy

    def close(self):
        if self.pool is not None:
            B.la_free_pool(self.pool)
        B.la_free_kv(self.kv)
        B.la_free_model(self.model)
        self.pool = self.kv = self.model = None

    # -- cache ----------------------------------------------------------------------
    def fill_kv(self, layer: int, k: np.ndarray, v: np.ndarray, row0: int = 0):
        kd, vd = B.to_device(k), B.to_device(v)
        B.la_kv_fill(self.kv, layer, row0, kd, vd)
        torch.cuda.synchronize()

    def read_kv(self, layer: int, row0: int, n: int):
        sh = self.shape
        dt = {"f32": torch.float32, "bf16": torch.int16, "f16": torch.float16}[sh.dtype]
        k = torch.empty((n, sh.n_kv_heads, sh.head_dim), dtype=dt, device="cuda")
        v = torch.empty_like(k)
        B.la_kv_read(self.kv, layer, row0, n, k, v)
        torch.cuda.synchronize()
        k, v = k.cpu().numpy(), v.cpu().numpy()
        if sh.dtype == "bf16":
            k, v = k.view(np.uint16), v.view(np.uint16)
        return k, v

    # -- single calls on numpy inputs (tests) -----------------------------------------
    def forward(self, hidden: np.ndarray, pos, vis, layer_begin=0, layer_end=None) -> np.ndarray:
        le = self.shape.n_layers if layer_end is None else layer_end
        h = B.to_device(np.asarray(hidden, dtype=np.float32))
        p = B.to_device(np.asarray(pos, dtype=np.int32))
        m = B.to_device(np.asarray([int(x) for x in vis], dtype=np.uint64))
        B.la_forward_layers(self.model, layer_begin, le, h, p, m, self.kv)
        torch.cuda.synchronize()
        return h.cpu().numpy()

    def unembed_argmax(self, hidden: np.ndarray):
        h = B.to_device(np.asarray(hidden, dtype=np.float32))
        ids = torch.empty(h.shape[0], dtype=torch.int32, device="cuda")
        top2 = torch.empty((h.shape[0], 2), dtype=torch.float32, device="cuda")
        B.la_unembed_argmax(self.model, h, ids, top2)
        torch.cuda.synchronize()
        return ids.cpu().numpy(), top2.cpu().numpy()

    # -- generation -------------------------------------------------------------------
    def prefill(self, tokens: np.ndarray, L0: int = 0):
        """Runs tokens through all layers (la_prefill: causal chunks inside the library); cache rows L0.. are filled."""
        toks = B.to_device(np.asarray(tokens, dtype=np.int32))
        B.la_prefill(self.model, self.kv, toks, L0)
        torch.cuda.synchronize()
        return L0 + len(tokens)

    def start(self, prompt: np.ndarray, W: int, N: int, G: int, Bp: int, seed_pool: bool = True,
              prefill: bool = True, sampling: dict | None = None):
        """Prefills prompt[:-1] (unless the cache rows are already there) and initialises the
        controller (pool, window, first block).  sampling: see generate."""
        if self.pool is not None:
            B.la_free_pool(self.pool)
        self.la = (W, N, G)
        self.Bp = Bp
        self.pool = B.la_pool_alloc(self.shape.vocab, N, G)
        self.state = B.new_state()
        if prefill:
            self.prefill(np.asarray(prompt[:-1]))
        B.la_state_init(self.pool, self.kv, W, N, G, B.to_device(np.asarray(prompt, dtype=np.int32)), Bp,
                        seed_pool, self.state)
        torch.cuda.synchronize()
        sh = self.shape
        self._hidden = torch.empty((Bp, sh.d_model), dtype=torch.float32, device="cuda")
        self._ids = torch.empty(Bp, dtype=torch.int32, device="cuda")
        self._top2 = torch.empty((Bp, 2), dtype=torch.float32, device="cuda")
        self._tok = B.state_field(self.state, "tok")[:Bp]
        self._pos = B.state_field(self.state, "pos")[:Bp]
        self._vis = B.state_field(self.state, "vis")[:Bp]
        # (a row's position is below max_len + Bp: guesses reach past the last token that fits)
        self._sample = None if sampling is None else self._sampler(sampling, Bp, self.max_len + Bp)

    def _sampler(self, sampling: dict, rows: int, n_u: int):
        """choose(hidden, ids, u_index) of rows that are all sampled alike: sampling = {temperature, top_k, top_p, min_p (each may be left out), and u, the random
        numbers, or seed}.  n_u: random numbers needed."""
        how = dict(sampling)
        u, seed = how.pop("u", None), how.pop("seed", 0)
        if u is None:
            u = torch.rand(n_u, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda")
        u = torch.as_tensor(u, dtype=torch.float32, device="cuda").flatten().contiguous()
        if u.numel() < n_u:
            raise ValueError(f"{u.numel()} random numbers, {n_u} needed")
        unknown = set(how) - {"temperature", "top_k", "top_p", "min_p"}
        if unknown:
            raise TypeError(f"unknown sampling parameters {sorted(unknown)}")
        rows_of = {k: torch.full((rows,), v, dtype=torch.int32 if k == "top_k" else torch.float32, device="cuda") for k, v in how.items() if v is not None}
        logits = torch.empty((rows, self.shape.vocab), dtype=torch.float32, device="cuda")

        def choose(hidden, ids, u_index):
            B.la_unembed_logits(self.model, hidden, logits)
            B.la_sample(logits, u, ids, u_index=u_index, **rows_of)

        return choose

    def _choose(self):
        """The block's ids: the largest logit of every row, or a sample drawn by the random number of the row's position, so that rows of one position and
        prefix, in whatever block, draw the same token."""
        if self._sample is None:
            B.la_unembed_argmax(self.model, self._hidden, self._ids, self._top2)
        else:
            self._sample(self._hidden, self._ids, self._pos)

    def step(self, emitted: torch.Tensor, max_total: int):
        """One decode step, enqueued without any host synchronisation."""
        W, N, G = self.la
        sh = self.shape
        B.la_embed(self.model, self._tok, self._hidden)
        B.la_forward_layers(self.model, 0, sh.n_layers, self._hidden, self._pos, self._vis, self.kv)
        self._choose()
        B.la_ngram_accept(self.pool, self.kv, W, N, G, self._ids, self.state, emitted, max_total)

    def generate(self, prompt: np.ndarray, n_new: int, W: int, N: int, G: int, Bp: int | None = None,
                 seed_pool: bool = True, poll: int = 8, sampling: dict | None = None):
        """Greedy generation; {W=0, N=1, G=0} is sequential decoding.  Returns (tokens, stats).
        sampling = {temperature, top_k, top_p, min_p, u or seed}: every token is sampled, the one behind position t with u[t] (max_len + Bp numbers; made from the
        seed if left out).  A candidate is accepted where it is the token that its row draws, so lookahead and sequential decoding emit the same tokens, but for rounding: with 16-bit
        weights a row's last bits go by the block that it stands in, and a number that falls on a border between two tokens may draw either (about one token in a thousand of the small
        test models; greedy decoding parts at near-ties alike)."""
        rows = 1 + (W + G) * (N - 1)
        Bp = rows if Bp is None else Bp
        self.start(prompt, W, N, G, Bp, seed_pool, sampling=sampling)
        emitted = torch.zeros(n_new, dtype=torch.int32, device="cuda")
        n_field = B.state_field(self.state, "n_emitted")
        done = 0
        while done < n_new:
            for _ in range(poll):
                self.step(emitted, n_new)
            done = int(n_field.item())
        st = B.read_state(self.state)
        if st.error:
            raise B.LaError(-4 if st.error & 4 else -3, f"a kernel raised error word {st.error} during generation")
        return emitted.cpu().numpy().astype(np.int64), dict(steps=st.steps, matched_steps=st.matched_steps,
                                                            n_emitted=st.n_emitted, L=st.L)

    # -- several requests at once -----------------------------------------------------------------
    def generate_batch(self, prompts, n_new: int, page_size: int = 16, n_pages: int | None = None, sampling: dict | None = None):
        """Sequential generation of n_new tokens for up to 64 prompts together, a token of each per step, on a cache of pages that they share (n_pages: as many as they need if
        left out); the contiguous cache takes one prompt after the other on its way there.  sampling: as in generate, the numbers as u[step][request].  Returns (tokens [requests, n_new], stats)."""
        sh, R, dev = self.shape, len(prompts), "cuda"
        prompts = [np.asarray(p, dtype=np.int32) for p in prompts]
        if not 1 <= R <= B.LA_MAX_ROWS or any(len(p) < 1 for p in prompts):
            raise ValueError(f"need 1 to {B.LA_MAX_ROWS} prompts of one token at least")
        lens = [len(p) - 1 for p in prompts]
        pages_of = lambda n: (n + page_size - 1) // page_size
        blocks = max(1, max(pages_of(n + n_new) for n in lens))
        need = max(1, sum(pages_of(n + n_new) for n in lens))
        n_pages = need if n_pages is None else n_pages
        if n_pages < need:  # (requests only grow here: what the last step needs is known)
            raise B.LaError(-3, f"the batch needs {need} pages of {page_size} positions, there are {n_pages}")
        i32 = lambda n, v=0: torch.full(n if isinstance(n, tuple) else (n,), v, dtype=torch.int32, device=dev)
        dt = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}[sh.dtype]
        pages = B.la_pages(*(torch.empty((sh.n_layers, n_pages, sh.n_kv_heads, page_size, sh.head_dim), dtype=dt, device=dev) for _ in range(2)))
        table, ring = i32((R, blocks), -1), torch.arange(n_pages, dtype=torch.int32, device=dev)
        heads, heads_out = torch.tensor([0, n_pages, 0, 0], dtype=torch.int32, device=dev), i32(4)
        old, new = i32(R), torch.tensor(lens, dtype=torch.int32, device=dev)

        def mapped(rows, error=None):  # pages and slots of the lengths `new`
            nonlocal heads, heads_out
            slot, pos, req, first = i32(rows), i32(rows), i32(rows), i32(R + 1)
            B.la_page_map(old, new, page_size, table, ring, heads, heads_out, slot, pos, req, first)
            heads, heads_out = heads_out, heads
            if error is not None:
                torch.maximum(error, heads[3:], out=error)
            return slot, pos, req

        def check(error):
            if int(error):
                raise B.LaError(-3, f"the pages do not hold the batch (error {int(error)} of la_page_map; {n_pages} pages of {page_size} positions)")

        # prompts one after the other through the contiguous cache, and from there into their pages
        error = i32(1)
        if sum(lens):
            slot, _, _ = mapped(sum(lens), error)
            check(error)
            at = 0
            for p in prompts:
                n = len(p) - 1
                if n:
                    self.prefill(p[:-1])
                    k = torch.empty((n, sh.n_kv_heads, sh.head_dim), dtype=dt, device=dev)
                    v = torch.empty_like(k)
                    for l in range(sh.n_layers):
                        B.la_kv_read(self.kv, l, 0, n, k, v)
                        B.la_paged_write(pages, l, k, v, slot[at:at + n])
                at += n
        choose = None if sampling is None else self._sampler(sampling, R, n_new * R)
        which = torch.arange(R, dtype=torch.int32, device=dev)
        hidden = torch.empty((R, sh.d_model), dtype=torch.float32, device=dev)
        ids, tokens = torch.tensor([p[-1] for p in prompts], dtype=torch.int32, device=dev), i32((n_new, R))
        for step in range(n_new):
            old.copy_(new)
            new.add_(1)
            slot, pos, req = mapped(R, error)
            B.la_embed(self.model, ids, hidden)
            B.la_forward_paged(self.model, 0, sh.n_layers, hidden, pos, req, slot, pages, table)
            ids = tokens[step]
            if choose is None:
                B.la_unembed_argmax(self.model, hidden, ids)
            else:
                choose(hidden, ids, which)
                which = which + R
        check(error)
        old.copy_(new)
        new.zero_()
        mapped(R, error)
        check(error)
        return tokens.t().cpu().numpy().astype(np.int64), dict(steps=n_new, pages=n_pages, free_pages=int(heads[1]))

    # -- the split deployment on one GPU, with an injected round trip ---------------------------------
    def step_split(self, emitted: torch.Tensor, max_total: int, head_layers: int, tail_layers: int, rtt_ms: float):
        """One decode step cut where the paper cuts the model (Section 3.1): the first
        `head_layers` and the last `tail_layers` layers are the local half, the layers between
        them the cloud half; the hidden states cross the cut twice per step, and each crossing
        costs half of rtt_ms here (a host sleep after the stream has drained, as a network would
        make the next half wait).  Returns (local_ms, cloud_ms) of GPU time, by host clock."""
        W, N, G = self.la
        n = self.shape.n_layers
        t0 = time.perf_counter()
        B.la_embed(self.model, self._tok, self._hidden)
        B.la_forward_layers(self.model, 0, head_layers, self._hidden, self._pos, self._vis, self.kv)
        torch.cuda.synchronize()
        t1 = time.perf_counter()
        time.sleep(rtt_ms / 2000.0)
        t2 = time.perf_counter()
        B.la_forward_layers(self.model, head_layers, n - tail_layers, self._hidden, self._pos, self._vis, self.kv)
        torch.cuda.synchronize()
        t3 = time.perf_counter()
        time.sleep(rtt_ms / 2000.0)
        t4 = time.perf_counter()
        B.la_forward_layers(self.model, n - tail_layers, n, self._hidden, self._pos, self._vis, self.kv)
        self._choose()
        B.la_ngram_accept(self.pool, self.kv, W, N, G, self._ids, self.state, emitted, max_total)
        torch.cuda.synchronize()
        t5 = time.perf_counter()
        return ((t1 - t0) + (t5 - t4)) * 1e3, (t3 - t2) * 1e3

    def generate_split(self, prompt: np.ndarray, n_new: int, W: int, N: int, G: int, head_layers: int, tail_layers: int,
                       rtt_ms: float, Bp: int | None = None, seed_pool: bool = True):
        """Greedy generation through step_split.  Returns (tokens, stats): steps, tokens per
        step, wall milliseconds per step, local and cloud GPU milliseconds per step, and the
        measured throughput, from which la_rtt_fixed_overhead / la_rtt_project give the paper's
        decomposition and projection (Section 6.3)."""
        rows = 1 + (W + G) * (N - 1)
        Bp = rows if Bp is None else Bp
        self.start(prompt, W, N, G, Bp, seed_pool)
        emitted = torch.zeros(n_new, dtype=torch.int32, device="cuda")
        n_field = B.state_field(self.state, "n_emitted")
        steps, local, cloud = 0, 0.0, 0.0
        t0 = time.perf_counter()
        while int(n_field.item()) < n_new:
            l, c = self.step_split(emitted, n_new, head_layers, tail_layers, rtt_ms)
            local += l
            cloud += c
            steps += 1
        wall = (time.perf_counter() - t0) * 1e3
        st = B.read_state(self.state)
        if st.error:
            raise B.LaError(-4 if st.error & 4 else -3, f"a kernel raised error word {st.error} during generation")
        return emitted.cpu().numpy().astype(np.int64), dict(
            steps=steps, tokens_per_step=n_new / steps, ms_per_step=wall / steps, local_ms=local / steps,
            cloud_ms=cloud / steps, tok_per_s=n_new / (wall / 1e3), matched_steps=st.matched_steps)

    # -- Jacobi decoding (Section 4.2) ------------------------------------------------------------------
    def generate_jacobi(self, prompt: np.ndarray, n_new: int, k: int, Bp: int | None = None, poll: int = 8):
        """Greedy generation by Jacobi iteration on blocks of k positions.  Returns (tokens, stats):
        passes (each one network round trip in the split deployment), blocks committed, tokens per pass."""
        Bp = k if Bp is None else Bp
        sh = self.shape
        self.state = B.new_state()
        self.prefill(np.asarray(prompt[:-1]))
        B.la_jacobi_init(self.kv, k, B.to_device(np.asarray(prompt, dtype=np.int32)), Bp, self.state)
        hidden = torch.empty((Bp, sh.d_model), dtype=torch.float32, device="cuda")
        ids = torch.empty(Bp, dtype=torch.int32, device="cuda")
        tok = B.state_field(self.state, "tok")[:Bp]
        pos = B.state_field(self.state, "pos")[:Bp]
        vis = B.state_field(self.state, "vis")[:Bp]
        emitted = torch.zeros(n_new, dtype=torch.int32, device="cuda")
        n_field = B.state_field(self.state, "n_emitted")
        done = 0
        while done < n_new:
            for _ in range(poll):
                B.la_embed(self.model, tok, hidden)
                B.la_forward_layers(self.model, 0, sh.n_layers, hidden, pos, vis, self.kv)
                B.la_unembed_argmax(self.model, hidden, ids)
                B.la_jacobi_accept(self.kv, k, ids, self.state, emitted, n_new)
            done = int(n_field.item())
        st = B.read_state(self.state)
        if st.error:
            raise B.LaError(-4 if st.error & 4 else -3, f"a kernel raised error word {st.error} during generation")
        return emitted.cpu().numpy().astype(np.int64), dict(passes=st.steps, blocks=st.matched_steps, n_emitted=st.n_emitted,
                                                            L=st.L, tokens_per_pass=n_new / max(st.steps, 1))
