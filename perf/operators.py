"""Operators between a prompt and its first token: chunks of new tokens whose
keys and values are written to the paged cache (in 32, 16 or 8 bits) and read
back, the attention of such a chunk over the paged cache, and sampling with
temperature, top-k, top-p and min-p from given uniforms.

`run` computes them in elementary torch operations, or, with `own`, through
the framework's entry points, on the same inputs.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

#: Query heads, KV heads, head dims, RoPE base and vocabulary of the shapes the framework is configured for.
LAYOUTS = {"8b": (32, 8, 128, 5e5, 128256), "7b": (28, 4, 128, 1e6, 152064), "1b": (16, 8, 128, 5e5, 128256),
           "tiny": (4, 4, 64, 1e4, 2048)}
BLOCK = 16                  # tokens of a cache block
E4M3_MAX = 448.0
SCALE_MIN, SCALE_MAX = -112, 119  # powers of two that a head row of an 8-bit cache may be scaled by


# --------------------------------------------------------------------------
# The cases
# --------------------------------------------------------------------------
def listed():
    return [
        # The rows of one decoding step of a middle batch go to an 8-bit cache: a launch or two is all there is.
        {"name": "store_8b_decode_b64", "op": "store", "layout": "8b", "cache": "e4m3", "B": 64, "chunk": 1, "ctx": 768,
         "spread": 0.5, "single": 0},
        # One prompt of ordinary length enters an empty 8-bit cache (its end inside a block).
        {"name": "store_8b_prompt2000", "op": "store", "layout": "8b", "cache": "e4m3", "B": 1, "chunk": 2000, "ctx": 0,
         "spread": 0.0, "single": 0},
        # A batch's whole 8-bit contexts read back, as when requests leave for another pool.
        {"name": "load_7b_b32", "op": "load", "layout": "7b", "cache": "e4m3", "B": 32, "chunk": 1500, "ctx": 0,
         "spread": 0.5, "single": 0},
        # The fp32 model that deployments are checked with: two short chunks.
        {"name": "attn_tiny_b2", "op": "attn", "layout": "tiny", "cache": "f32", "B": 2, "chunk": 24, "ctx": 40,
         "spread": 0.2, "single": 0},
        # Plain decoding of a middle batch over an 8-bit cache: bound by reading it.
        {"name": "attn_8b_decode_b64", "op": "attn", "layout": "8b", "cache": "e4m3", "B": 64, "chunk": 1, "ctx": 768,
         "spread": 0.5, "single": 0},
        # A long prompt in one chunk (bf16 cache): matrix work.
        {"name": "attn_8b_prompt4096", "op": "attn", "layout": "8b", "cache": "bf16", "B": 1, "chunk": 4096, "ctx": 0,
         "spread": 0.0, "single": 0},
        # A middle chunk of a long prompt over what is cached of it in 8 bits.
        {"name": "attn_8b_chunk512", "op": "attn", "layout": "8b", "cache": "e4m3", "B": 1, "chunk": 512, "ctx": 8000,
         "spread": 0.0, "single": 0},
        # A mixed batch of a serving loop: most sequences decode, some are in their prompts (seven query heads a KV head).
        {"name": "attn_7b_mixed_b24", "op": "attn", "layout": "7b", "cache": "bf16", "B": 24, "chunk": 250, "ctx": 1500,
         "spread": 0.5, "single": 16},
        # One request's next token: latency.
        {"name": "sample_8b_b1", "op": "sample", "layout": "8b", "rows": 1, "temperature": 0.8, "top_k": 50, "top_p": 0.9,
         "min_p": 0.0, "hot": 9.0, "mixed": False, "probs": False},
        # A draft position of a middle batch, with the truncated distribution that the acceptance test divides by.
        {"name": "sample_8b_b61_q", "op": "sample", "layout": "8b", "rows": 61, "temperature": 0.7, "top_k": 0,
         "top_p": 0.95, "min_p": 0.0, "hot": 9.0, "mixed": False, "probs": True},
        # A large batch whose requests each bring settings of their own (some greedy, some not truncated at all).
        {"name": "sample_7b_b256_mixed", "op": "sample", "layout": "7b", "rows": 256, "temperature": 1.0, "top_k": 200,
         "top_p": 0.9, "min_p": 0.02, "hot": 7.0, "mixed": True, "probs": False},
        # The check model's small vocabulary.
        {"name": "sample_tiny_b5", "op": "sample", "layout": "tiny", "rows": 5, "temperature": 1.2, "top_k": 0,
         "top_p": 0.8, "min_p": 0.05, "hot": 4.0, "mixed": False, "probs": True},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49))))))


def draw(rng):
    op = rng.choice(["store", "store", "load", "attn", "attn", "attn", "attn", "sample", "sample", "sample"])
    if op == "sample":
        layout = rng.choice(["8b", "7b", "7b", "tiny"])
        return {"op": op, "layout": layout, "rows": _log_int(rng, 1, 256), "temperature": rng.choice([0.3, 0.6, 0.8, 1.0, 1.5]),
                "top_k": rng.choice([0, 1, _log_int(rng, 2, 2000)]), "top_p": rng.choice([1.0, 0.5, round(rng.uniform(0.7, 0.99), 3)]),
                "min_p": rng.choice([0.0, 0.0, round(rng.uniform(0.01, 0.2), 3)]), "hot": rng.choice([3.0, 7.0, 9.0, 11.0]),
                "mixed": rng.random() < 0.3, "probs": rng.random() < 0.4 and layout != "7b"}
    layout = rng.choice(["8b", "7b", "1b", "tiny"])
    cache = "f32" if layout == "tiny" else rng.choice(["bf16", "e4m3", "e4m3"])
    spread = rng.choice([0.0, 0.3, 0.5])
    B = _log_int(rng, 1, 64)
    single = rng.choice([0, 0, B // 2, B])
    if layout == "tiny":
        return {"op": op, "layout": layout, "cache": cache, "B": min(B, 8), "chunk": _log_int(rng, 1, 60), "ctx": _log_int(rng, 1, 200),
                "spread": spread, "single": min(single, 8)}
    # what a case costs grows with its rows (and, for attention, with the keys they see)
    chunk = _log_int(rng, 1, max(1, 2000 // B))
    ctx = _log_int(rng, 1, 8000 if chunk <= 64 else 2000)
    if op == "attn":
        ctx = min(ctx, 60000 // B)
    return {"op": op, "layout": layout, "cache": cache, "B": B, "chunk": chunk, "ctx": ctx, "spread": spread, "single": single}


# --------------------------------------------------------------------------
# Inputs
# --------------------------------------------------------------------------
class State:
    pass


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(gen, *shape):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32)


def _dev(a, dtype=torch.int32):
    return torch.as_tensor(np.ascontiguousarray(a)).to(device="cuda", dtype=dtype)


def _lengths(case, seed):
    """New tokens and cached tokens of each sequence: the same lengths for every seed, in another order."""
    r = np.random.default_rng(0)
    B, s = case["B"], case["spread"]
    n = np.clip(np.rint(case["chunk"] * np.exp(s * r.standard_normal(B))), 1, 3 * case["chunk"]).astype(np.int64)
    n[:case["single"]] = 1
    c = np.clip(np.rint(case["ctx"] * np.exp(s * r.standard_normal(B))), 0, 3 * case["ctx"]).astype(np.int64)
    p = np.random.default_rng(seed).permutation(B)
    return n[p], c[p]


def _table(total, seed):
    """Blocks of each sequence, from a shuffled pool with a few to spare; -1 where there is none."""
    need = -(-total // BLOCK)
    pool = int(need.sum() * 1.05) + 2
    perm = np.random.default_rng(seed + 1).permutation(pool)
    table = np.full((len(total), int(need.max())), -1, np.int32)
    at = 0
    for b, k in enumerate(need):
        table[b, :k] = perm[at:at + k]
        at += k
    return table, pool


def _quantise(x):
    """e4m3 codes and scale bytes of fp32 head rows [..., D]: the smallest power of two that brings a row's largest
    finite magnitude to 448 or less."""
    amax = torch.where(torch.isfinite(x), x.abs(), torch.zeros_like(x)).amax(-1)
    f, e = torch.frexp(amax)
    e = torch.where(f <= 0.875, e - 9, e - 8)
    e = torch.where(amax == 0, torch.full_like(e, SCALE_MIN), e).clamp(SCALE_MIN, SCALE_MAX)
    down = ((127 - e) << 23).to(torch.int32).view(torch.float32)  # 2^-e
    y = x * down[..., None]
    y = torch.where(torch.isfinite(y), y.clamp(-E4M3_MAX, E4M3_MAX), torch.full_like(y, math.nan))
    return y.to(torch.float8_e4m3fn).view(torch.uint8), (e + 127).to(torch.uint8)


def _values(codes, scales):
    """The values that codes [..., D] with scale bytes [...] stand for, in fp32 (exact)."""
    up = (scales.to(torch.int32) << 23).view(torch.float32)
    return codes.view(torch.float8_e4m3fn).to(torch.float32) * up[..., None]


def _hot_logits(gen, rows, vocab, hot):
    """Logits as language models give them: a broad bulk, and a few tokens far above it."""
    l = 2.2 * _normal(gen, rows, vocab)
    ids = torch.randint(0, vocab, (rows, min(200, vocab // 8)), generator=gen, device="cuda")
    return l.scatter_add_(1, ids, hot + 2.0 * _normal(gen, *ids.shape))


def _inputs(case, seed):
    """The tensors of a case (a dict), the same whoever computes on them."""
    gen, op = _gen(seed), case["op"]
    H, Hkv, D, theta, V = LAYOUTS[case["layout"]]
    if op == "sample":
        R = case["rows"]
        i = {"logits": _hot_logits(gen, R, V, case["hot"]), "u": torch.rand(R, generator=gen, device="cuda", dtype=torch.float32)}
        t, k, p, m = (np.full(R, case[n]) for n in ("temperature", "top_k", "top_p", "min_p"))
        if case["mixed"]:  # every request its own
            r = np.random.default_rng(seed + 2)
            t = t * r.choice([0.0, 0.5, 0.8, 1.0, 1.3], R)
            k = k * r.choice([0, 1, 1, 4], R)
            p = np.where(r.random(R) < 0.4, 1.0, p)
            m = m * r.choice([0.0, 0.0, 1.0, 3.0], R)
        return i | {"t": _dev(t, torch.float32), "k": _dev(k), "p": _dev(p, torch.float32), "m": _dev(m, torch.float32)}
    n, c = _lengths(case, seed)
    table, pool = _table(n + c, seed)
    rows, starts = int(n.sum()), np.concatenate([[0], np.cumsum(n)])
    i = {"n": n, "c": c, "starts": _dev(starts), "ctx": _dev(c), "table": _dev(table), "pool": pool, "rows": rows}
    cache = case["cache"]
    kt = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.uint8}[cache]
    if op == "store":
        # K has a few dims that are much larger than the others, as trained models' keys do
        x = _normal(gen, rows, H + 2 * Hkv, D)
        x[:, H:H + Hkv, 3::31] *= 6.0
        x[:, H + Hkv:] *= 0.5
        i["qkv"] = x.view(rows, -1)
        k, v = torch.zeros((pool, Hkv, BLOCK, D), dtype=kt, device="cuda"), torch.zeros((pool, Hkv, D, BLOCK), dtype=kt, device="cuda")
        ks, vs = (torch.full((pool, Hkv, BLOCK), 127, dtype=torch.uint8, device="cuda") for _ in range(2))
    else:
        k, v = 0.8 * _normal(gen, pool, Hkv, BLOCK, D), 0.5 * _normal(gen, pool, Hkv, BLOCK, D)
        ks = vs = None
        if cache == "e4m3":
            (k, ks), (v, vs) = _quantise(k), _quantise(v)
        v = v.transpose(2, 3)
        k, v = k.to(kt).contiguous(), v.to(kt).contiguous()
        if op == "attn":
            i["q"] = _normal(gen, rows, H, D).to(torch.float32 if cache == "f32" else torch.bfloat16)
    return i | {"k": k, "v": v, "ks": ks if cache == "e4m3" else None, "vs": vs if cache == "e4m3" else None}


def prepare(case, seed):
    st = State()
    st.case, st.op = case, case["op"]
    st.H, st.Hkv, st.D, st.theta, st.V = LAYOUTS[case["layout"]]
    st.__dict__.update({"i": _inputs(case, seed)})
    i, rows = st.i, case.get("rows") or st.i["rows"]
    st.out = torch.float32 if case.get("cache") in (None, "f32") else torch.bfloat16
    if st.op == "sample":
        st.tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
        st.probs = torch.empty((rows, st.V), dtype=torch.float32, device="cuda") if case["probs"] else None
    else:
        st.longest = int((i["n"] + i["c"]).max())
        st.q_out = torch.empty((rows, st.H, st.D), dtype=st.out, device="cuda")
        st.k_out, st.v_out = (torch.empty((rows, st.Hkv, st.D), dtype=st.out, device="cuda") for _ in range(2))
    if own:
        from paper_2512_22420_amd import device, workload
        st.dev = device
        if st.op == "sample":
            st.ws = device.sample_workspace(rows, st.V)
        else:
            shape = {"8b": workload.LLAMA8B_LAYER, "7b": workload.QWEN7B, "1b": workload.LLAMA1B_DRAFT,
                     "tiny": workload.TINY_F32}[case["layout"]]
            st.desc = device.model_desc(shape)
            st.layer = device.KvLayer(i["k"], i["v"], i["ks"], i["vs"])
            st.batch = device.ChunkBatch(i["starts"], i["ctx"], i["table"], rows, int(i["n"].max()))
            st.ws = device.chunk_workspace(st.desc, st.batch)
    return st


# --------------------------------------------------------------------------
# One pass
# --------------------------------------------------------------------------
def run(st):
    if own:
        return _run_own(st)
    return {"store": _store, "load": _load, "attn": _attn, "sample": _sample}[st.op](st)


def _run_own(st):
    dev, i = st.dev, st.i
    if st.op == "sample":
        dev.sample(i["logits"], i["u"], st.tokens, st.ws, temperature=i["t"], top_k=i["k"], top_p=i["p"], min_p=i["m"], probs=st.probs)
        return {"tokens": st.tokens} if st.probs is None else {"tokens": st.tokens, "probs": st.probs}
    if st.op == "attn":
        dev.chunk_attn(st.desc, st.layer, st.batch, i["q"], st.q_out, st.ws)
        return {"o": st.q_out}
    if st.op == "store":
        dev.chunk_store(st.desc, st.layer, st.batch, i["qkv"], st.ws, q_out=st.q_out)
    dev.chunk_load(st.desc, st.layer, st.batch, st.k_out, st.v_out, st.ws)
    return {"k": st.k_out, "v": st.v_out} | ({"q": st.q_out} if st.op == "store" else {})


def _places(st):
    """Position, block and slot of every row of the chunk."""
    i = st.i
    r = torch.arange(i["rows"], device="cuda")
    seq = torch.searchsorted(i["starts"].long(), r, right=True) - 1
    pos = i["ctx"].long()[seq] + r - i["starts"].long()[seq]
    return seq, pos, i["table"].long()[seq, pos // BLOCK], pos % BLOCK


def _rows_of(st, blk, slot):
    """K and V [.., Hkv, D] in fp32 of the cached tokens at (blk, slot)."""
    i = st.i
    k, v = i["k"][blk, :, slot], i["v"].transpose(2, 3)[blk, :, slot]
    if i["ks"] is None:
        return k.float(), v.float()
    return _values(k, i["ks"][blk, :, slot]), _values(v, i["vs"][blk, :, slot])


def _store(st):
    i, H, Hkv, D = st.i, st.H, st.Hkv, st.D
    _, pos, blk, slot = _places(st)
    x = i["qkv"].view(i["rows"], H + 2 * Hkv, D)
    # 64 bits: the angle of a far position, and a key next to a border between two codes
    freq = st.theta ** (-2.0 * torch.arange(D // 2, device="cuda", dtype=torch.float64) / D)
    ang = pos.double()[:, None] * freq
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    a, b = x[:, :H + Hkv, :D // 2].double(), x[:, :H + Hkv, D // 2:].double()
    qk = torch.cat([a * c - b * s, b * c + a * s], -1).float()
    k, v = qk[:, H:], x[:, H + Hkv:]
    if i["ks"] is not None:
        k, ks = _quantise(k)
        v, vs = _quantise(v)
        i["ks"][blk, :, slot], i["vs"][blk, :, slot] = ks, vs
    i["k"][blk, :, slot] = k.to(i["k"].dtype)
    i["v"].transpose(2, 3)[blk, :, slot] = v.to(i["v"].dtype)
    return _load(st) | {"q": qk[:, :H].to(st.out)}


def _load(st):
    _, _, blk, slot = _places(st)
    k, v = _rows_of(st, blk, slot)
    return {"k": k.to(st.out), "v": v.to(st.out)}


def _attn(st):
    i, H, Hkv, D = st.i, st.H, st.Hkv, st.D
    B, N, L, G = len(i["n"]), int(i["n"].max()), st.longest, H // Hkv
    starts, ctx = i["starts"].long(), i["ctx"].long()
    t = torch.arange(L, device="cuda")
    blk = i["table"].long()[:, t // BLOCK].clamp(min=0)                       # [B, L]
    k, v = _rows_of(st, blk, (t % BLOCK).expand(B, L))                          # [B, L, Hkv, D]
    j = torch.arange(N, device="cuda")
    row = (starts[:B, None] + j).clamp(max=i["rows"] - 1)                       # [B, N]
    q = i["q"][row].float().view(B, N, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B * Hkv, G * N, D)
    k, v = (x.permute(0, 2, 1, 3).reshape(B * Hkv, L, D) for x in (k, v))
    s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(B, Hkv, G, N, L) / math.sqrt(D)
    s.masked_fill_((t > (ctx[:, None] + j)[..., None])[:, None, None], -math.inf)
    s = (s - s.amax(-1, keepdim=True)).exp_()
    o = torch.matmul(s.view(B * Hkv, G * N, L), v).view(B, Hkv, G, N, D) / s.sum(-1, keepdim=True)
    seq, pos, _, _ = _places(st)
    return {"o": o.permute(0, 3, 1, 2, 4)[seq, pos - ctx[seq]].reshape(i["rows"], H, D).to(st.out)}


def _sample(st):
    # 64 bits: sums over a whole vocabulary, and a token is one side of a border or the other
    i = st.i
    l, greedy = i["logits"], (i["t"] == 0)[:, None]
    order = torch.sort(l, dim=-1, descending=True, stable=True)
    T = torch.where(greedy, 1.0, i["t"][:, None].double())
    w = torch.exp((order.values.double() - order.values[:, :1].double()) / T)
    rank = torch.arange(l.shape[1], device="cuda")
    k = torch.where(i["k"] <= 0, l.shape[1], i["k"])[:, None]
    w = w * (rank < torch.where(greedy, 1, k))
    target = i["p"][:, None].double() * w.sum(-1, keepdim=True)
    before = w.cumsum(-1) - w
    w = w * (((before < target) | (i["p"][:, None] >= 1) | (rank == 0)) & (w >= i["m"][:, None].double()))
    w = torch.zeros_like(w).scatter_(1, order.indices, w)
    run_ = w.cumsum(-1)
    total = run_[:, -1:]
    j = (run_ <= i["u"][:, None].double() * total).sum(-1)
    last = l.shape[1] - 1 - (w.flip(-1) > 0).int().argmax(-1)
    tokens = torch.minimum(j, last).int()
    return {"tokens": tokens} if not st.case["probs"] else {"tokens": tokens, "probs": (w / total).float()}


# --------------------------------------------------------------------------
# What a pass cannot do without
# --------------------------------------------------------------------------
def work(case):
    H, Hkv, D, _, V = LAYOUTS[case["layout"]]
    if case["op"] == "sample":
        R = case["rows"]
        return {"bytes": R * V * 4 * (2 if case["probs"] else 1) + R * 24, "flops": R * V * 4}
    n, c = _lengths(case, 0)
    rows, e = int(n.sum()), {"f32": 4, "bf16": 2, "e4m3": 1}[case["cache"]]
    out = 4 if case["cache"] == "f32" else 2
    token = 2 * Hkv * (D * e + (1 if e == 1 else 0))  # K and V of one cached token
    if case["op"] == "attn":
        keys = int((n * c + n * (n + 1) // 2).sum())
        return {"bytes": 2 * rows * H * D * out + int((n + c).sum()) * token, "flops": 4 * H * D * keys}
    load = {"bytes": rows * (token + 2 * Hkv * D * out), "flops": rows * 2 * Hkv * D}
    if case["op"] == "load":
        return load
    return {"bytes": rows * ((H + 2 * Hkv) * D * 4 + H * D * out + token) + load["bytes"],
            "flops": rows * (H + Hkv) * D * 3 + load["flops"]}


# --------------------------------------------------------------------------
# The same from the definitions, in 64 bits
# --------------------------------------------------------------------------
def _e4m3_grid():
    """The magnitudes of e4m3 from its definition, as float64, by code."""
    code = np.arange(127)
    ex, man = code >> 3, code & 7
    return np.where(ex == 0, man / 8 * 2.0 ** -6, (1 + man / 8) * 2.0 ** (ex - 7.0))


def _nearest_e4m3(x):
    """x [.., D] (float64) -> the value its 8-bit form stands for: scaled by the row's power of two, rounded to the
    nearest code, ties to the even one."""
    grid = torch.as_tensor(_e4m3_grid(), device=x.device)
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.clamp(amax, min=1e-300) / E4M3_MAX))
    e = torch.where(amax > E4M3_MAX * 2.0 ** e, e + 1, e)
    e = torch.where(amax <= E4M3_MAX * 2.0 ** (e - 1), e - 1, e).clamp(SCALE_MIN, SCALE_MAX)
    y = x / 2.0 ** e
    m = y.abs().clamp(max=E4M3_MAX)
    hi = torch.searchsorted(grid, m.contiguous()).clamp(max=126)
    lo = (hi - 1).clamp(min=0)
    dl, dh = m - grid[lo], grid[hi] - m
    pick = torch.where((dl < dh) | ((dl == dh) & (lo % 2 == 0)), lo, hi)
    return torch.sign(y) * grid[pick] * 2.0 ** e


def _cached(i, b, count):
    """K and V [Hkv, count, D] of sequence b's first `count` cached tokens, in float64."""
    blocks = i["table"][b, : -(-count // BLOCK)].long()
    got = []
    for pages, scale, order in ((i["k"], i["ks"], (1, 0, 2, 3)), (i["v"], i["vs"], (1, 0, 3, 2))):
        x = pages[blocks].permute(*order)  # [Hkv, blocks, 16, D]
        if scale is not None:
            u = x.long()
            grid = torch.as_tensor(_e4m3_grid(), device="cuda")
            x = torch.where(u >= 128, -1.0, 1.0).double() * grid[(u & 127).clamp(max=126)]
            x = x * 2.0 ** (scale[blocks].permute(1, 0, 2).double() - 127)[..., None]
        got.append(x.double().reshape(x.shape[0], -1, x.shape[-1])[:, :count])
    return got


def exact(case, seed):
    i = _inputs(case, seed)
    H, Hkv, D, theta, V = LAYOUTS[case["layout"]]
    if case["op"] == "sample":
        return _exact_sample(case, i)
    first = i["starts"].tolist()
    if case["op"] == "attn":
        out = []
        for b, (n, c) in enumerate(zip(i["n"].tolist(), i["c"].tolist())):
            K, Vv = _cached(i, b, n + c)
            q = i["q"][first[b]:first[b] + n].double()
            o = torch.empty((n, H, D), dtype=torch.float64, device="cuda")
            for r0 in range(0, n, 512):
                r1 = min(n, r0 + 512)
                hidden = torch.arange(n + c, device="cuda")[None] > c + torch.arange(r0, r1, device="cuda")[:, None]
                for h in range(H):
                    g = h // (H // Hkv)
                    s = (q[r0:r1, h] @ K[g].T) * D ** -0.5
                    o[r0:r1, h] = torch.softmax(s.masked_fill(hidden, -math.inf), -1) @ Vv[g]
            out.append(o)
        return {"o": torch.cat(out)}
    if case["op"] == "load":
        kv = [_cached(i, b, n) for b, n in enumerate(i["n"].tolist())]  # these chunks begin at position 0
        if i["c"].any():
            kv = [[x[:, c:] for x in _cached(i, b, n + c)] for b, (n, c) in enumerate(zip(i["n"].tolist(), i["c"].tolist()))]
        return {"k": torch.cat([x[0].transpose(0, 1) for x in kv]), "v": torch.cat([x[1].transpose(0, 1) for x in kv])}
    pos = torch.cat([torch.arange(c, c + n, device="cuda", dtype=torch.float64) for n, c in zip(i["n"].tolist(), i["c"].tolist())])
    x = i["qkv"].double().view(i["rows"], H + 2 * Hkv, D)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"),
                       pos[:, None] * torch.exp(torch.arange(0, D, 2, device="cuda", dtype=torch.float64) * (-math.log(theta) / D)))
    z = torch.complex(x[:, :H + Hkv, :D // 2], x[:, :H + Hkv, D // 2:]) * turn[:, None]
    qk = torch.cat([z.real, z.imag], -1)
    k, v = qk[:, H:], x[:, H + Hkv:]
    if case["cache"] == "e4m3":
        k, v = _nearest_e4m3(k), _nearest_e4m3(v)
    return {"q": qk[:, :H], "k": k, "v": v}


def _exact_sample(case, i):
    l, u, t, k, p, m = (i[n].double().cpu().numpy() for n in ("logits", "u", "t", "k", "p", "m"))
    tokens, probs = np.empty(len(l), np.int32), np.zeros(l.shape) if case["probs"] else None
    for r, row in enumerate(l):
        order = np.argsort(-row, kind="stable")
        if t[r] == 0:
            order = order[:1]
        elif k[r] > 0:
            order = order[:int(k[r])]
        w = np.exp((row[order] - row[order[0]]) / (t[r] or 1.0))
        if p[r] < 1:
            many = 1 + int(np.searchsorted(np.cumsum(w), p[r] * math.fsum(w)))
            order, w = order[:many], w[:many]
        order, w = order[w >= m[r]], w[w >= m[r]]
        by = np.argsort(order)
        order, c = order[by], np.cumsum(w[by])
        tokens[r] = order[min(int(np.searchsorted(c, u[r] * c[-1], side="right")), len(order) - 1)]
        if probs is not None:
            probs[r, order] = w[by] / c[-1]
    return {"tokens": tokens} if probs is None else {"tokens": tokens, "probs": probs}
