"""The chunk calls and the sampler as a serving loop uses them together: prompts
enter the cache and decoding goes on from there, the verify step reads pages that
chunks have filled, and the sampler's distributions feed the acceptance test."""
import dataclasses

import numpy as np
import pytest
import torch

import serve_ref as ref
from paper_2512_22420_amd import binding as nb
from paper_2512_22420_amd import workload as W
from paper_2512_22420_amd.device import (ChunkBatch, KvLayer, Scratch, chunk_attn, chunk_load, chunk_store,
                                        chunk_workspace, device_error, model_desc, pack_weight, sample, sample_workspace)

pytestmark = pytest.mark.gpu

BF = dataclasses.replace(W.LLAMA8B_LAYER, n_heads=8, n_kv_heads=2, d_model=1024, vocab=4096)
F32 = W.TINY_F32


def _stream():
    return torch.cuda.current_stream().cuda_stream


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a)).to("cuda", torch.int32)


def _pages(shape, pages, pool):
    dt = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.uint8}[pages]
    s = shape
    k = torch.zeros((pool, s.n_kv_heads, 16, s.head_dim), dtype=dt, device="cuda")
    v = torch.zeros((pool, s.n_kv_heads, s.head_dim, 16), dtype=dt, device="cuda")
    sc = [torch.full((pool, s.n_kv_heads, 16), 127, dtype=torch.uint8, device="cuda") for _ in range(2)] if pages == "e4m3" else [None] * 2
    return KvLayer(k, v, *sc)


class Matmul:
    """x @ w.T to fp32: the framework's GEMM for bf16, torch for the fp32 check model."""

    def __init__(self, shape, w, M):
        N, K = w.shape
        self.bf = shape.dtype == "bf16"
        self.w, self.size, self.y = w, (M, N, K), torch.empty((M, N), device="cuda")
        if self.bf:
            self.packed = pack_weight(w.to(torch.bfloat16).view(torch.int16))
            self.ws = Scratch(nb.gemm_workspace_bytes(nb.NJ_BF16, M, N, K, nb.NJ_GEMM_STORE))

    def __call__(self, x):
        if not self.bf:
            return torch.mm(x.float(), self.w.t(), out=self.y)
        M, N, K = self.size
        nb.gemm(nb.NJ_BF16, x.data_ptr(), self.packed.data_ptr(), self.y.data_ptr(), M, N, K, nb.NJ_GEMM_STORE, self.ws.ptr,
                self.ws.nbytes, _stream())
        return self.y


class Decoder:
    """One attention layer between an embedding and an LM head, with its cache."""

    def __init__(self, shape, pages, prompts, steps, seed):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        s, B = shape, len(prompts)
        self.shape, self.pages, self.B, self.desc = s, pages, B, model_desc(s)
        dt = torch.bfloat16 if s.dtype == "bf16" else torch.float32
        width = (s.n_heads + 2 * s.n_kv_heads) * s.head_dim
        self.embed = torch.randn((s.vocab, s.d_model), generator=g, device="cuda").to(dt)
        w_qkv = torch.randn((width, s.d_model), generator=g, device="cuda") * s.d_model ** -0.5
        w_out = torch.randn((s.vocab, s.n_heads * s.head_dim), generator=g, device="cuda") * 3 * (s.n_heads * s.head_dim) ** -0.5
        rows = sum(prompts)
        need = [-(-(p + steps) // 16) for p in prompts]
        perm = np.random.default_rng(seed).permutation(sum(need) + 2)
        table, at = np.full((B, max(need)), -1, np.int32), 0
        for b, n in enumerate(need):
            table[b, :n] = perm[at:at + n]
            at += n
        self.layer, self.table = _pages(s, pages, len(perm)), _i32(table)
        self.ctx, self.one = torch.zeros(B, dtype=torch.int32, device="cuda"), _i32(np.arange(B + 1))
        self.prompt_len = _i32(prompts)
        self.prompt = ChunkBatch(_i32(np.concatenate([[0], np.cumsum(prompts)])), self.ctx, self.table, rows, max(prompts))
        self.step = ChunkBatch(self.one, self.ctx, self.table, B, 1)
        self.calls = {}
        for name, batch in (("prompt", self.prompt), ("step", self.step)):
            M = batch.rows
            self.calls[name] = (batch, Matmul(s, w_qkv, M), chunk_workspace(self.desc, batch),
                                torch.empty((M, s.n_heads, s.head_dim), dtype=dt, device="cuda"),
                                torch.empty((M, s.n_heads * s.head_dim), dtype=dt, device="cuda"))
        self.head, self.sws = Matmul(s, w_out, B), sample_workspace(B, s.vocab)
        self.tokens, self.u = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, device="cuda")
        f = lambda *v: torch.tensor((v * B)[:B], device="cuda")  # noqa: E731
        self.T, self.p, self.m = f(0.8, 0.0, 1.0, 1.3, 0.6), f(0.9, 1.0, 1.0, 0.95, 0.5), f(0.0, 0.0, 0.02, 0.0, 0.0)
        self.k = _i32(np.resize([40, 0, 0, 7, 1], B))
        self.probs = torch.empty((B, s.vocab), device="cuda")

    def attend(self, name, tokens):
        """The chunk's attention output rows."""
        batch, qkv, ws, q, out = self.calls[name]
        x = self.embed[tokens.long()]
        chunk_store(self.desc, self.layer, batch, qkv(x), ws, q_out=q)
        chunk_attn(self.desc, self.layer, batch, q, out, ws)
        return out

    def draw(self, rows):
        sample(self.head(rows), self.u, self.tokens, self.sws, temperature=self.T, top_k=self.k, top_p=self.p, min_p=self.m,
               probs=self.probs)

    def errors(self):
        return [device_error(ws) for ws in (self.calls["prompt"][2], self.calls["step"][2], self.sws)]

    def values(self, b, n):
        """K and V [n, Hkv, D] (float64) as they stand in the pages."""
        blk, slot = self.table[b].cpu().numpy().astype(np.int64)[np.arange(n) // 16], np.arange(n) % 16
        got = []
        for pages, sc in ((self.layer.k, self.layer.k_scale), (self.layer.v.transpose(2, 3), self.layer.v_scale)):
            x = pages[torch.as_tensor(blk).cuda(), :, torch.as_tensor(slot).cuda()].cpu()
            got.append(x.double().numpy() if sc is None else ref.decode(x.numpy(), sc.cpu().numpy()[blk, :, slot]))
        return got


def _check_rows(dec, q, out, k, v, ctx):
    """Rows of one sequence against the 64-bit reference; the tolerance counts p's and the output's rounding to bf16
    (2^-8 of sum p |v| and of the output) and fp32 sums of up to D + 2 and ctx + n + 8 terms."""
    D = dec.shape.head_dim
    o, a, big = ref.attention(q.double().cpu().numpy(), k, v, ctx)
    half = 2.0 ** -8 if dec.shape.dtype == "bf16" else 0.0
    soft = 2 * (D + 2) * 2.0 ** -24 * big + (len(k) + 8) * 2.0 ** -24
    tol = 1.02 * (half * (a + np.abs(o)) + soft * a) + 2.0 ** -23 * np.abs(o)
    assert (np.abs(out.double().cpu().numpy().reshape(o.shape) - o) <= tol).all()


@pytest.mark.parametrize("pages,shape", [("e4m3", BF), ("bf16", BF), ("f32", F32)], ids=["e4m3", "bf16", "f32"])
def test_prompts_then_decoding(pages, shape):
    """Ragged prompts in one chunk, then eight tokens drawn one by one: every stored key and value, every attention row
    and every token against the reference, the decoding steps run eagerly and replayed from a graph."""
    prompts, steps = [37, 1, 16, 250, 5], 8
    toks = torch.randint(0, shape.vocab, (sum(prompts),), generator=torch.Generator().manual_seed(3)).cuda()
    us = np.random.default_rng(5).random((steps + 1, len(prompts))).astype(np.float32)
    runs = []
    for graphed in (False, True):
        dec = Decoder(shape, pages, prompts, steps, seed=1)
        starts = dec.prompt.starts.cpu().numpy()
        out = dec.attend("prompt", toks)
        qkv = dec.calls["prompt"][1].y.cpu().numpy().reshape(len(toks), -1, shape.head_dim)
        q = dec.calls["prompt"][3]
        H, Hkv = shape.n_heads, shape.n_kv_heads
        for b, n in enumerate(prompts):
            r = slice(starts[b], starts[b + 1])
            k, v = dec.values(b, n)
            kk = ref.rotate(qkv[r, H:H + Hkv], np.arange(n), shape.rope_theta).astype(np.float32)
            # half a step of the page's type; e4m3: of the largest codes' spacing (2^5 of 448) where the row is scaled
            for got, x in ((k, kk), (v, qkv[r, H + Hkv:])):
                size = np.abs(x).max(-1, keepdims=True)
                tol = {"f32": 2.0 ** -23 * np.abs(x), "bf16": 2.0 ** -8 * np.abs(x) * 1.01, "e4m3": 2.0 ** -4 * np.abs(x) * 1.01 + size * 2.0 ** -17}[pages]
                assert (np.abs(got - x) <= tol).all()
            _check_rows(dec, q[r], out[r], k, v, 0)
        last = (dec.prompt.starts[1:] - 1).long()
        dec.ctx.copy_(dec.prompt_len)
        dec.u.copy_(torch.as_tensor(us[0]))
        dec.draw(out[last].contiguous())

        def step():
            dec.draw(dec.attend("step", dec.tokens))
            dec.ctx.add_(1)
        got = [dec.tokens.clone()]
        if graphed:  # warmed up and captured on a state that is put back
            keep = [t.clone() for t in (dec.ctx, dec.tokens)]
            step()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                step()
            dec.ctx.copy_(keep[0])
            dec.tokens.copy_(keep[1])
        for i in range(steps - 1):
            dec.u.copy_(torch.as_tensor(us[i + 1]))
            if graphed:
                graph.replay()
            else:
                step()
                _, _, _, q, out = dec.calls["step"]
                logits = dec.head.y.cpu().numpy()
                for b, n in enumerate(prompts):
                    _check_rows(dec, q[b:b + 1], out[b:b + 1], *dec.values(b, n + i + 1), n + i)
                    f = lambda t: float(t[b].cpu())  # noqa: E731
                    want, pr = ref.sample(logits[b], f(dec.u), f(dec.T), int(f(dec.k)), f(dec.p), f(dec.m))
                    assert int(dec.tokens[b]) == want
                    assert (np.abs(dec.probs[b].cpu().numpy() - pr) <= (2.0 ** -23 + shape.vocab * 2.0 ** -44) * pr + 2.0 ** -149).all()
            got.append(dec.tokens.clone())
        total = [n + steps - 1 for n in prompts]
        rows = ChunkBatch(_i32(np.concatenate([[0], np.cumsum(total)])), torch.zeros_like(dec.ctx), dec.table, sum(total), max(total))
        back = [torch.empty((sum(total), Hkv, shape.head_dim), dtype=q.dtype, device="cuda") for _ in range(2)]
        ws = Scratch(256)
        chunk_load(dec.desc, dec.layer, rows, *back, ws)
        at = np.concatenate([[0], np.cumsum(total)])
        for b, n in enumerate(total):
            for x, want in zip(back, dec.values(b, n)):
                assert np.array_equal(x[at[b]:at[b + 1]].double().cpu().numpy(), want)
        assert dec.errors() == [0, 0, 0] and device_error(ws) == 0
        runs.append((torch.stack(got), back[0], back[1]))
    for a, b in zip(*runs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("shape,k", [(BF, 3), (BF, 15), (W.QWEN7B, 4), (F32, 3)], ids=["bf16-k3", "bf16-k15", "7b-k4", "f32-k3"])
def test_verify_attention_reads_pages_that_chunks_filled(shape, k):
    """A window's attention by nightjar_attn_verify over contexts that chunk_store wrote, and by chunk_attn with the
    window stored too: the same rows to both calls' rounding."""
    s, T = dataclasses.replace(shape, n_layers=1), k + 1
    lens = np.array([90, 1, 33, 16])
    B, desc = len(lens), model_desc(s)
    rng = np.random.default_rng(7)
    width = s.n_heads + 2 * s.n_kv_heads
    starts = np.concatenate([[0], np.cumsum(lens)])
    need = -(-(lens + T) // 16)
    table = np.full((B, need.max()), -1, np.int32)
    perm, at = rng.permutation(need.sum()), 0
    for b in range(B):
        table[b, :need[b]] = perm[at:at + need[b]]
        at += need[b]
    bf = s.dtype == "bf16"
    layer, table, dt = _pages(s, "bf16" if bf else "f32", int(need.sum())), _i32(table), torch.bfloat16 if bf else torch.float32
    x = torch.as_tensor(rng.standard_normal((int(lens.sum()), width * s.head_dim)).astype(np.float32)).cuda()
    prompt = ChunkBatch(_i32(starts), _i32(np.zeros(B)), table, len(x), int(lens.max()))
    window = ChunkBatch(_i32(np.arange(B + 1) * T), _i32(lens), table, B * T, T)
    ws = chunk_workspace(desc, prompt)
    ws2 = chunk_workspace(desc, window)
    chunk_store(desc, layer, prompt, x, ws)
    y = torch.as_tensor(rng.standard_normal((B * T, width * s.head_dim)).astype(np.float32)).cuda()
    q = torch.empty((B * T, s.n_heads, s.head_dim), dtype=dt, device="cuda")
    # the window's rows as the cache would hold them, from pages of their own
    own = KvLayer(torch.zeros_like(layer.k), torch.zeros_like(layer.v))
    chunk_store(desc, own, window, y, ws2, q_out=q)
    kw, vw = (torch.empty((B * T, s.n_kv_heads, s.head_dim), dtype=dt, device="cuda") for _ in range(2))
    chunk_load(desc, own, window, kw, vw, ws2)
    win_k = torch.zeros((B, s.n_kv_heads, 16, s.head_dim), dtype=dt, device="cuda")
    win_v = torch.zeros((B, s.n_kv_heads, s.head_dim, 16), dtype=dt, device="cuda")
    win_k[:, :, :T] = kw.view(B, T, s.n_kv_heads, -1).transpose(1, 2)
    win_v[:, :, :, :T] = vw.view(B, T, s.n_kv_heads, -1).permute(0, 2, 3, 1)
    n = nb.attn_workspace_bytes(desc, B, k)
    vws = Scratch(n)
    a, b = (torch.empty((B * T, s.n_heads * s.head_dim), dtype=dt, device="cuda") for _ in range(2))
    nb.attn_verify(desc, q.data_ptr(), layer.k.data_ptr(), layer.v.data_ptr(), layer.k.shape[0], win_k.data_ptr(), win_v.data_ptr(),
                   table.data_ptr(), table.shape[1], window.context_lens.data_ptr(), B, k, a.data_ptr(), vws.ptr, n, _stream())
    chunk_store(desc, layer, window, y, ws2)
    chunk_attn(desc, layer, window, q, b, ws2)
    assert [device_error(w) for w in (ws, ws2, vws)] == [0, 0, 0]
    for i, ctx in enumerate(lens):
        r = slice(i * T, (i + 1) * T)
        blk, slot = table[i].long()[torch.arange(ctx + T).cuda() // 16], torch.arange(ctx + T).cuda() % 16
        kk, vv = layer.k[blk, :, slot].double().cpu().numpy(), layer.v.transpose(2, 3)[blk, :, slot].double().cpu().numpy()
        o, mag, big = ref.attention(q[r].double().cpu().numpy(), kk, vv, int(ctx))
        half = 2.0 ** -8 if bf else 0.0
        tol = 1.02 * (half * (mag + np.abs(o)) + (2 * (s.head_dim + 2) * 2.0 ** -24 * big + (len(kk) + 8) * 2.0 ** -24) * mag) + 2.0 ** -23 * np.abs(o)
        assert (np.abs(b[r].double().cpu().numpy().reshape(o.shape) - o) <= tol).all()
        # the verify kernel's p may be rounded too, and its reference may lag a row's max: twice p's part
        assert (np.abs((a[r].double() - b[r].double()).cpu().numpy().reshape(o.shape)) <= 3 * tol).all()


def test_truncated_distributions_in_the_acceptance_test():
    """A draft drawn with top-k and top-p, its distributions as draft_probs, the target's truncated ones as logits
    (their logarithm): accepted lengths and tokens as the rule says, in 64 bits, and no token outside the target's."""
    B, k, V = 24, 3, 5000
    rng = np.random.default_rng(11)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    target = torch.randn((B, k + 1, V), generator=g, device="cuda") * 3
    draft = (target[:, :k] + 0.7 * torch.randn((B, k, V), generator=g, device="cuda")).contiguous()
    full = lambda v, dt=torch.float32: torch.full((B,), v, dtype=dt, device="cuda")  # noqa: E731
    q = torch.empty((B, k, V), device="cuda")
    toks = torch.empty((k, B), dtype=torch.int32, device="cuda")
    ws = sample_workspace(B * (k + 1), V)
    for i in range(k):  # column i of the draft: rows a stride of k * V apart
        u = torch.rand(B, generator=g, device="cuda")
        sample(draft[:, i], u, toks[i], ws, temperature=full(0.9), top_k=full(60, torch.int32), top_p=full(0.9), probs=q[:, i])
    p = torch.empty((B * (k + 1), V), device="cuda")
    spare, R = torch.empty(B * (k + 1), dtype=torch.int32, device="cuda"), B * (k + 1)
    sample(target.view(R, V), torch.rand(R, generator=g, device="cuda"), spare, ws,
           temperature=torch.full((R,), 0.9, device="cuda"), top_p=torch.full((R,), 0.8, device="cuda"), probs=p)
    assert device_error(ws) == 0
    drafts = toks.t().contiguous()
    u = torch.as_tensor(rng.random((B, k + 1)).astype(np.float32)).cuda()
    logits = torch.log(p).view(B, k + 1, V).contiguous()
    desc = model_desc(dataclasses.replace(F32, vocab=V))
    aws = Scratch(nb.accept_workspace_bytes(V, B, k))
    acc, nxt = torch.full((B,), -7, dtype=torch.int32, device="cuda"), torch.full((B, k + 1), -7, dtype=torch.int32, device="cuda")
    nb.accept(desc, logits.data_ptr(), drafts.data_ptr(), q.data_ptr(), u.data_ptr(), B, k, acc.data_ptr(), nxt.data_ptr(),
              aws.ptr, aws.nbytes, _stream())
    assert device_error(aws) == 0
    pt, qd, dr, uu = p.view(B, k + 1, V).double().cpu().numpy(), q.double().cpu().numpy(), drafts.cpu().numpy(), u.double().cpu().numpy()
    acc, nxt = acc.cpu().numpy(), nxt.cpu().numpy()
    checked = 0
    for b in range(B):
        assert (qd[b, np.arange(k), dr[b]] > 0).all()  # every draft token has a share in its distribution
        n, near = 0, False
        while n < k:
            ratio = pt[b, n, dr[b, n]] / qd[b, n, dr[b, n]]
            near |= abs(uu[b, n] - min(1.0, ratio)) < 1e-5  # (fp32 on the other side of a border is no mistake)
            if not uu[b, n] < min(1.0, ratio):
                break
            n += 1
        last = nxt[b, acc[b]]
        assert (nxt[b, :acc[b]] == dr[b, :acc[b]]).all() and pt[b, acc[b], last] > 0
        if not near:
            assert acc[b] == n
            checked += 1
    assert checked > B // 2 and 0 < acc.mean() < k


def test_two_graphs_on_one_workspace():
    """Two captured calls that share a workspace, replayed in turn: each gives its eager result every time (the counters
    that join parts of cut keys are left as they were found)."""
    s = dataclasses.replace(W.LLAMA8B_LAYER, n_heads=16, n_kv_heads=4)
    desc = model_desc(s)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    cases = []
    for lens, n in (([5000, 40], [1, 3]), ([1200], [70])):
        total = np.asarray(lens) + n
        need = -(-total // 16)
        table = np.full((len(lens), need.max()), -1, np.int32)
        at = 0
        for b, c in enumerate(need):
            table[b, :c] = np.arange(at, at + c)
            at += c
        k, v = (torch.randn(sh, generator=g, device="cuda").to(torch.bfloat16) for sh in ((at, 4, 16, 128), (at, 4, 128, 16)))
        rows = sum(n)
        batch = ChunkBatch(_i32(np.concatenate([[0], np.cumsum(n)])), _i32(lens), _i32(table), rows, max(n))
        cases.append((KvLayer(k, v), batch, torch.randn((rows, 16, 128), generator=g, device="cuda").to(torch.bfloat16),
                      torch.empty((rows, 2048), dtype=torch.bfloat16, device="cuda")))
    ws = Scratch(max(nb.chunk_attn_workspace_bytes(desc, c[1].B, c[1].rows, c[1].max_chunk) for c in cases))
    want, graphs = [], []
    for layer, batch, q, out in cases:
        chunk_attn(desc, layer, batch, q, out, ws)
        want.append(out.clone())
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            chunk_attn(desc, layer, batch, q, out, ws)
    for rep in range(4):
        for i in ((0, 1), (1, 0))[rep % 2]:
            cases[i][3].zero_()
            graphs[i].replay()
        torch.cuda.synchronize()
        for c, w in zip(cases, want):
            assert torch.equal(c[3], w)
            chunk_attn(desc, c[0], c[1], c[2], c[3], ws)
    assert device_error(ws) == 0


def test_tensors_off_the_gpu_are_refused():
    l, u, t, ws = torch.zeros((2, 8), device="cuda"), torch.zeros(2), torch.zeros(2, dtype=torch.int32, device="cuda"), sample_workspace(2, 8)
    with pytest.raises(TypeError, match="GPU"):
        sample(l, u, t, ws)
    desc, layer = model_desc(F32), _pages(F32, "f32", 2)
    out = [torch.zeros((3, 4, 64), device=d) for d in ("cuda", "cpu")]
    for where in ("cuda", "cpu"):
        batch = ChunkBatch(*(torch.tensor(x, dtype=torch.int32, device=where) for x in ([0, 3], [0], [[0]])), 3, 3)
        with pytest.raises(TypeError, match="GPU"):
            chunk_load(desc, layer, batch, out[0], out[int(where == "cuda")], Scratch(256))
