"""Cases that measure the attention half of a decoder layer on one GPU: attention over a paged cache with a shared prefix
(``ls_paged_kv_attend``), the append to that cache with the position rotation (``ls_paged_kv_append``), and the norms before
and after a block with gate and residual scale (``ls_block_norm``).

Each operator is here in three forms: its plain form in 32 bits (``own`` false), the framework's call (``own`` true), and its
definition in 64 bits (``exact``).  Head counts and widths are those of the stacks this package is benchmarked on (7B, 13B and
70B decoders, head size 128) and generic ones.
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "f32": torch.float32}
DEV = "cuda"


# ---- the cases --------------------------------------------------------------------------------------------------------------
def _attend(name, dtype, heads, kv_heads, seqs, prefix, suffix, page, layout="token", head_dim=128, q_len=1, window=0, idle=0):
    return {"name": name, "op": "attend", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "seqs": seqs,
            "q_len": q_len, "prefix": prefix, "suffix": suffix, "window": window, "idle": idle, "page": page, "layout": layout}


def _append(name, dtype, heads, kv_heads, seqs, chunk, rope_dim, page, layout="token", head_dim=128, interleaved=False, fused=True):
    return {"name": name, "op": "append", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "seqs": seqs,
            "chunk": chunk, "rope_dim": rope_dim, "interleaved": interleaved, "fused": fused, "page": page, "layout": layout}


def _norm(name, tokens, width, residual, block, post, gain, gate, scale):
    return {"name": name, "op": "norm", "tokens": tokens, "width": width, "residual": residual, "block": block, "post": post,
            "gain": gain, "gate": gate, "scale": scale}


def listed():
    return [
        # one user's next token early in a conversation: latency
        _attend("attend 1 short", "bf16", 32, 8, 1, 0, 333, 16),
        # one user's next token over a long document: the cache is all there is to read
        _attend("attend 1 long", "bf16", 64, 8, 1, 0, 100001, 64, "head"),
        # samples drawn from one prompt, as many key heads as query heads; the prompt does not end with a page
        _attend("attend 33 samples", "fp16", 40, 40, 33, 1500, 500, 16),
        # four draft tokens verified per sequence under a sliding window, some slots of the batch empty
        _attend("attend drafts window", "fp16", 32, 8, 16, 1000, 6000, 32, q_len=4, window=4096, idle=2),
        # a serving batch on a long few-shot prefix: prefix work and own caches of similar size
        _attend("attend 128 few-shot", "bf16", 64, 8, 128, 8192, 1024, 64),
        # a batch of questions about one very long document: matrix products over the shared prefix
        _attend("attend 64 document", "bf16", 64, 8, 64, 65536, 1024, 128, "head"),
        # one token of one sequence: latency
        _append("append 1", "bf16", 32, 8, 1, 1, 128, 16),
        # a decode step of a batch at scattered positions, half of each head rotated, pairs side by side
        _append("append 200 partial", "fp16", 64, 8, 200, 1, 64, 64, "head", interleaved=True),
        # chunks of prompts
        _append("append chunks", "bf16", 64, 8, 16, 1023, 128, 16),
        # one token between blocks, the residual in 32 bits: latency
        _norm("norm 1", 1, 4096, "f32", "bf16", False, False, "none", 1.0),
        # a decode batch with norms on both sides, a gate for each channel and a residual scale, odd width
        _norm("norm 200 odd", 200, 5121, "f32", "fp16", True, True, "channel", 0.5),
        # a prompt, residual in 16 bits, a gate for each token and channel
        _norm("norm prompt", 8192, 8192, "bf16", "bf16", True, True, "token", 0.22),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "append", "norm"])
    most = [work(c) for c in listed() if c["op"] == op]
    while True:
        if op == "norm":
            width = 8 * (_log(rng, 8, 1024) | 1) if rng.random() < 0.7 else _log(rng, 64, 8192) | 1
            c = _norm("", _log(rng, 1, 16384), width, rng.choice(["f32", "f32", "bf16", "fp16"]), rng.choice(["bf16", "fp16"]), rng.random() < 0.6,
                      rng.random() < 0.6, rng.choice(["none", "channel", "token"]), rng.choice([1.0, 0.5, 0.22]))
            if c["residual"] != "f32":
                c["block"] = c["residual"]
        else:
            heads, kv_heads = rng.choice([(32, 32), (32, 8), (40, 40), (64, 8), (16, 2), (8, 1), (28, 4)])
            head_dim = rng.choice([128, 128, 64])
            dtype, layout, page = rng.choice(["bf16", "fp16"]), rng.choice(["token", "head"]), rng.choice([16, 24, 32, 64, 128])
            if op == "append":
                seqs = _log(rng, 1, 256)
                chunk = 1 if rng.random() < 0.5 else _log(rng, 2, 4096) | 1
                c = _append("", dtype, heads, kv_heads, seqs, chunk, rng.choice([0, head_dim // 2, head_dim, head_dim]), page, layout, head_dim,
                            rng.random() < 0.3, rng.random() < 0.7)
            else:
                seqs = _log(rng, 1, 256)
                prefix = rng.choice([0, page * (_log(rng, 1, 65536 // page) | 1), _log(rng, 17, 65536) | 1])
                q_len = rng.choice([1, 1, 1, 2, 5, 8])
                window = rng.choice([0, 0, 0, _log(rng, 64, 8192) | 1])
                idle = rng.choice([0, 0, 1]) if seqs > 2 else 0
                c = _attend("", dtype, heads, kv_heads, seqs, prefix, q_len + (_log(rng, 1, 32768) | 1), page, layout, head_dim, q_len, window, idle)
        c.pop("name")
        w = work(c)
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most) and _plain_bytes(c) <= 16e9:
            return c


def _plain_bytes(c):
    """What the plain attention holds at once, about: its scores and its copies of the own keys and values in 32 bits."""
    if c["op"] != "attend":
        return 0
    keys = c["prefix"] + c["suffix"] + c["page"]
    return 4 * c["seqs"] * (3 * c["q_len"] * c["heads"] * keys + 2 * (c["suffix"] + c["page"]) * c["kv_heads"] * c["head_dim"])


def _own_lengths(c):
    """Positions of its own (after the prefix) that each sequence has, between a quarter of the longest and the longest; the
    last ``idle`` slots are empty (-1 stands for a slot without a sequence)."""
    got = []
    for b in range(c["seqs"]):
        f = 1.0 if b == 0 else 0.25 + 0.75 * ((b * 0.6180339887) % 1.0)
        got.append(max(c["q_len"], int(round(c["suffix"] * f))) if b < c["seqs"] - c["idle"] else -1)
    return got


def work(c):
    if c["op"] == "norm":
        n, r, b = c["tokens"] * c["width"], 4 if c["residual"] == "f32" else 2, 2
        gate = {"none": 0, "channel": b * c["width"], "token": b * n}[c["gate"]]
        return {"bytes": n * (2 * r + 2 * b) + gate + (4 * c["width"] * (1 + c["post"]) if c["gain"] else 0), "flops": 10 * n}
    if c["op"] == "append":
        t, d = c["seqs"] * c["chunk"], c["head_dim"]
        return {"bytes": t * (2 * 2 * (c["heads"] + 2 * c["kv_heads"]) * d + 4 * c["rope_dim"] + 8),
                "flops": 3 * t * (c["heads"] + c["kv_heads"]) * c["rope_dim"]}
    lo_prefix, keys_own, pairs, rows = c["prefix"], 0, 0, 0
    for own_len in _own_lengths(c):
        if own_len < 0:
            continue
        end = c["prefix"] + own_len
        first = max(0, end - c["q_len"] + 1 - c["window"]) if c["window"] else 0
        lo_prefix, keys_own = min(lo_prefix, first), keys_own + end - max(first, c["prefix"])
        for i in range(c["q_len"]):
            p = end - c["q_len"] + 1 + i
            pairs += min(p, c["window"]) if c["window"] else p
        rows += c["q_len"]
    d = c["head_dim"]
    return {"bytes": (c["prefix"] - lo_prefix + keys_own) * c["kv_heads"] * d * 4 + c["seqs"] * c["q_len"] * c["heads"] * (4 * d + 4),
            "flops": 4 * d * c["heads"] * pairs}


# ---- the inputs -------------------------------------------------------------------------------------------------------------
class State:
    pass


def _randn(gen, shape, dtype, std=1.0):
    x = torch.empty(shape, dtype=dtype, device=DEV)
    return x.normal_(0.0, std, generator=gen)


def _pool(gen, c, n_pages):
    shape = (n_pages, c["page"], c["kv_heads"], c["head_dim"])
    if c["layout"] == "head":
        shape = (n_pages, c["kv_heads"], c["page"], c["head_dim"])
    k, v = (_randn(gen, shape, DTYPES[c["dtype"]]) for _ in range(2))
    return (k.transpose(1, 2), v.transpose(1, 2)) if c["layout"] == "head" else (k, v)


def _rope_table(positions, rope_dim):
    """Cosines, then sines, of position * 10000^(-2 i / rope_dim), computed in 64 bits and kept in 32."""
    i = torch.arange(rope_dim // 2, dtype=torch.float64, device=DEV)
    angle = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-2.0 * i / rope_dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def prepare(case, seed):
    c, s = case, State()
    s.case = c
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if c["op"] == "norm":
        _prepare_norm(c, s, gen)
    elif c["op"] == "append":
        _prepare_append(c, s, gen)
    else:
        _prepare_attend(c, s, gen, seed)
    return s


def _prepare_attend(c, s, gen, seed):
    page, dt = c["page"], DTYPES[c["dtype"]]
    lens = [c["prefix"] + n if n >= 0 else 0 for n in _own_lengths(c)]
    order = torch.randperm(c["seqs"], generator=torch.Generator().manual_seed(seed)).tolist()
    lens = [lens[j] for j in order]
    first, width = c["prefix"] // page, -(-(c["prefix"] + c["suffix"]) // page)
    n_prefix = -(-c["prefix"] // page)
    # pages of the pool are handed out in a shuffled order; a sequence holds its own copy of the page the prefix ends in
    need = [max(0, -(-n // page) - first) for n in lens]
    total = n_prefix + sum(need)
    ids = torch.randperm(total, generator=gen, device=DEV).to(torch.int32)
    s.k_pages, s.v_pages = _pool(gen, c, total)
    s.prefix_pages = ids[:n_prefix].clone()
    s.table = torch.zeros(c["seqs"], width, dtype=torch.int32, device=DEV)
    s.table[:, :n_prefix] = s.prefix_pages
    at = n_prefix
    for b, n in enumerate(need):
        s.table[b, first:first + n] = ids[at:at + n]
        at += n
    if c["prefix"] % page:  # the copies of the last, shared part of a page
        alive = torch.tensor([b for b, n in enumerate(lens) if n], device=DEV)
        to, part = s.table[alive, first].long(), c["prefix"] % page
        s.k_pages[to, :part] = s.k_pages[s.prefix_pages[first].long(), :part]
        s.v_pages[to, :part] = s.v_pages[s.prefix_pages[first].long(), :part]
    s.seq_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    # scores of trained models spread over several units: queries longer than unit variance
    s.q = _randn(gen, (c["seqs"], c["q_len"], c["heads"], c["head_dim"]), dt, 2.0)
    s.out = torch.empty_like(s.q)
    s.lse = torch.empty(c["seqs"], c["q_len"], c["heads"], dtype=torch.float32, device=DEV)
    if own:
        from paper_2609_03079_b200 import binding as ls
        s.kv = ls.ls_paged_kv_create(s.k_pages, s.v_pages, c["heads"], max_seqs=c["seqs"], max_q_len=c["q_len"])


def _prepare_append(c, s, gen):
    page, dt, T = c["page"], DTYPES[c["dtype"]], c["seqs"] * c["chunk"]
    limit = max(32768, 2 * c["chunk"])
    start = torch.randint(0, limit - c["chunk"], (c["seqs"],), generator=gen, device=DEV)
    per = -(-c["chunk"] // page) + 1
    ids = torch.randperm(c["seqs"] * per, generator=gen, device=DEV).to(torch.int32).view(c["seqs"], per)
    width = -(-limit // page) + 1
    s.table = torch.zeros(c["seqs"], width, dtype=torch.int32, device=DEV)
    s.table.scatter_(1, start[:, None] // page + torch.arange(per, device=DEV), ids)
    s.seq = torch.arange(c["seqs"], device=DEV, dtype=torch.int32).repeat_interleave(c["chunk"])
    s.pos = (start[:, None] + torch.arange(c["chunk"], device=DEV)).reshape(-1).to(torch.int32)
    s.k_pages, s.v_pages = _pool(gen, c, c["seqs"] * per)
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    if c["fused"]:  # slices of one projection's output
        s.q, s.k, s.v = _randn(gen, (T, h + 2 * g, d), dt).split([h, g, g], 1)
    else:
        s.q, s.k, s.v = (_randn(gen, (T, n, d), dt) for n in (h, g, g))
    s.q_out = torch.empty(T, h, d, dtype=dt, device=DEV)
    s.rope = _rope_table(limit, c["rope_dim"]) if c["rope_dim"] else None
    if own:
        from paper_2609_03079_b200 import binding as ls
        s.kv = ls.ls_paged_kv_create(s.k_pages, s.v_pages, h, rope=s.rope, rope_interleaved=c["interleaved"])


def _prepare_norm(c, s, gen):
    T, W, dt, dr = c["tokens"], c["width"], DTYPES[c["block"]], DTYPES[c["residual"]]
    s.x = _randn(gen, (T, W), dr, 2.0)
    s.x[:, :: max(1, W // 7)] *= 20.0  # a residual stream has a few large channels
    s.y = _randn(gen, (T, W), dt, 0.5)
    s.w_post = 1.0 + _randn(gen, (W,), torch.float32, 0.1) if c["gain"] and c["post"] else None
    s.w_pre = 1.0 + _randn(gen, (W,), torch.float32, 0.1) if c["gain"] else None
    s.gate = None if c["gate"] == "none" else _randn(gen, (W,) if c["gate"] == "channel" else (T, W), dt, 0.7)
    s.x_out, s.h = torch.empty_like(s.x), torch.empty_like(s.y)
    s.eps = 1e-5


# ---- one pass ---------------------------------------------------------------------------------------------------------------
def run(s):
    c = s.case
    if not own:
        return {"attend": _plain_attend, "append": _plain_append, "norm": _plain_norm}[c["op"]](s)
    from paper_2609_03079_b200 import binding as ls
    if c["op"] == "attend":
        ls.ls_paged_kv_attend(s.kv, s.q, s.out, s.seq_len, s.table, s.prefix_pages, c["prefix"], window=c["window"], lse=s.lse)
        return s.out, s.lse
    if c["op"] == "append":
        ls.ls_paged_kv_append(s.kv, s.q, s.k, s.v, s.q_out, s.seq, s.pos, s.table)
        return s.q_out, s.k_pages, s.v_pages
    ls.ls_block_norm(s.x, s.y, s.x_out, s.h, post_norm=c["post"], w_post=s.w_post, gate=s.gate, scale=c["scale"], w_pre=s.w_pre, eps=s.eps)
    return s.x_out, s.h


def _plain_attend(s):
    c, page = s.case, s.case["page"]
    B, n, H, D = s.q.shape
    P, first = c["prefix"], c["prefix"] // c["page"]
    q = s.q.float().view(B, n, c["kv_heads"], H // c["kv_heads"], D)
    kp, vp = (t[s.prefix_pages.long()].float().flatten(0, 1) for t in (s.k_pages, s.v_pages))
    ko, vo = (t[s.table[:, first:].long()].float().flatten(1, 2) for t in (s.k_pages, s.v_pages))
    at = torch.cat([torch.arange(kp.shape[0], device=DEV), torch.arange(ko.shape[1], device=DEV) + first * page])
    shared = torch.arange(at.numel(), device=DEV) < kp.shape[0]
    pos = s.seq_len[:, None] - n + torch.arange(n, device=DEV)
    seen = (at <= pos[..., None]) & (shared == (at < P))
    if c["window"]:
        seen &= at > pos[..., None] - c["window"]
    score = torch.cat([torch.einsum("bnhgd,khd->bnhgk", q, kp), torch.einsum("bnhgd,bkhd->bnhgk", q, ko)], -1) * D ** -0.5
    score = torch.where(seen[:, :, None, None], score, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(score.sub_(top))
    total = e.sum(-1, keepdim=True)
    ep, eo = e.split([kp.shape[0], ko.shape[1]], -1)
    out = torch.einsum("bnhgk,khd->bnhgd", ep, vp) + torch.einsum("bnhgk,bkhd->bnhgd", eo, vo)
    out = torch.where(total > 0, out / total, 0.0)
    lse = top + torch.log(total)
    return out.reshape(B, n, H, D).to(s.q.dtype), lse.reshape(B, n, H)


def _rotated(s, x):
    r = s.case["rope_dim"]
    x = x.float()
    if r == 0:
        return x
    cos, sin = s.rope[s.pos.long()].view(-1, 1, 2, r // 2).unbind(2)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if s.case["interleaved"] else (x[..., : r // 2], x[..., r // 2:r])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.stack(y, -1).flatten(-2) if s.case["interleaved"] else torch.cat(y, -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_append(s):
    page = s.case["page"]
    pos = s.pos.long()
    at = s.table[s.seq.long(), pos // page].long()
    s.k_pages[at, pos % page] = _rotated(s, s.k).to(s.k.dtype)
    s.v_pages[at, pos % page] = s.v
    s.q_out.copy_(_rotated(s, s.q))
    return s.q_out, s.k_pages, s.v_pages


def _plain_norm(s):
    def rms(z):
        return z * torch.rsqrt(z.square().mean(-1, keepdim=True) + s.eps)

    t = s.y.float()
    if s.case["post"]:
        t = rms(t)
    if s.w_post is not None:
        t = t * s.w_post
    if s.gate is not None:
        t = t * s.gate.float()
    x = s.x.float() + s.case["scale"] * t
    h = rms(x)
    if s.w_pre is not None:
        h = h * s.w_pre
    return x.to(s.x.dtype), h.to(s.y.dtype)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------
def exact(case, seed):
    c, s = case, prepare(case, seed)
    return {"attend": _exact_attend, "append": _exact_append, "norm": _exact_norm}[c["op"]](c, s)


def _exact_attend(c, s):
    """Sequence by sequence, all of its keys gathered, one softmax over what each token sees."""
    B, n, H, D = s.q.shape
    G, P, page = H // c["kv_heads"], c["prefix"], c["page"]
    out = torch.zeros(B, n, H, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, n, H), -math.inf, dtype=torch.float64, device=DEV)
    kp, vp = (t[s.prefix_pages.long()].double().flatten(0, 1)[:P] for t in (s.k_pages, s.v_pages))
    for b, length in enumerate(s.seq_len.tolist()):
        if length == 0:
            continue
        pages = s.table[b, P // page: -(-length // page)].long()
        ko, vo = (t[pages].double().flatten(0, 1)[P % page: length - P // page * page] for t in (s.k_pages, s.v_pages))
        k, v = torch.cat([kp, ko]).transpose(0, 1), torch.cat([vp, vo]).transpose(0, 1)  # [kv_heads, length, D]
        for i in range(n):
            end = length - n + i + 1
            begin = max(0, end - c["window"]) if c["window"] else 0
            score = s.q[b, i].double().view(-1, G, D) @ k[:, begin:end].transpose(1, 2) / math.sqrt(D)
            lse[b, i] = torch.logsumexp(score, -1).view(-1)
            out[b, i] = (torch.softmax(score, -1) @ v[:, begin:end]).view(H, D)
    return out, lse


def _exact_append(c, s):
    """As a product of complex numbers: (a + i b) e^{i angle}."""
    r = c["rope_dim"]

    def turned(x):
        x = x.double()
        if r == 0:
            return x
        t = s.rope[s.pos.long()].double()
        turn = torch.complex(t[:, : r // 2], t[:, r // 2:])[:, None]
        x, y = x.clone(), x
        first, second = (slice(0, r, 2), slice(1, r, 2)) if c["interleaved"] else (slice(0, r // 2), slice(r // 2, r))
        z = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        x[..., first], x[..., second] = z.real, z.imag
        return x

    k_pages, v_pages = s.k_pages.double(), s.v_pages.double()
    slot = s.pos.long() % c["page"]
    at = s.table[s.seq.long(), torch.div(s.pos, c["page"], rounding_mode="floor").long()].long()
    k_pages[at, slot], v_pages[at, slot] = turned(s.k), s.v.double()
    return turned(s.q), k_pages, v_pages


def _exact_norm(c, s):
    t = s.y.double()
    if c["post"]:
        t = t / (t.pow(2).mean(1, keepdim=True) + s.eps).sqrt()
    for factor in (s.w_post, s.gate):
        if factor is not None:
            t = t * factor.double()
    x = s.x.double() + c["scale"] * t
    h = x / (x.pow(2).mean(1, keepdim=True) + s.eps).sqrt()
    return x, h if s.w_pre is None else h * s.w_pre.double()
