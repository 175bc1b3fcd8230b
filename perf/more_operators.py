"""Cases that measure a key/value cache held in 4 bits on one GPU: storing new tokens in it, with the rotation by their positions
(``ls_paged_kv4_append``), reading tokens back in 16 bits (``ls_paged_kv4_read``), and the attention that reads it
(``ls_paged_kv4_attend``).

Each operator is here in three forms: its plain form in 32 bits (``own`` false), the framework's call (``own`` true), and its
definition in 64 bits (``exact``).  Head counts and widths are those of the stacks this package is benchmarked on (7B, 13B and
70B decoders, head size 128) and generic ones.

Every ``group`` components of a head's key (or value) share a scale and a zero of the cache's 16-bit type:
    x: the key as a 16-bit cache would hold it (turned in 64 bits, rounded to 32 and then 16), or the value as it is
    zero = min x;  scale = (max x - min x) / 15;  code = min(15, (x - zero) / scale to the nearest whole number, ties to even)
    what is held: scale * code + zero
A page holds tiles of 16 tokens for each key head, and a tile 16 rows of key codes, 16 of value codes, 16 of (scale, zero) of
keys, 16 of values.  Components stand in a code row in the order that the matrix instructions take them (``_order``).
"""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
DEV = "cuda"


# ---- the cases --------------------------------------------------------------------------------------------------------------
def _attend(name, dtype, heads, kv_heads, seqs, keys, page, group=64, head_dim=128, q_len=1, window=0, idle=0):
    return {"name": name, "op": "attend", "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "group": group, "seqs": seqs,
            "q_len": q_len, "keys": keys, "window": window, "idle": idle, "page": page}


def _tokens(name, op, dtype, heads, kv_heads, seqs, chunk, page, group=64, head_dim=128, rope_dim=0, interleaved=False, fused=True):
    return {"name": name, "op": op, "dtype": dtype, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "group": group, "seqs": seqs, "chunk": chunk,
            "rope_dim": rope_dim, "interleaved": interleaved, "fused": fused, "page": page}


def _store(name, *a, **kw):
    return _tokens(name, "store", *a, **kw)


def _read(name, *a, **kw):
    return _tokens(name, "read", *a, **kw)


def listed():
    return [
        # one user's next token early in a conversation: latency
        _attend("attend 1 short", "bf16", 32, 8, 1, 333, 16),
        # one user's next token over a long document: the cache is all there is to read
        _attend("attend 1 long", "bf16", 64, 8, 1, 100001, 64),
        # a batch of conversations, as many key heads as query heads
        _attend("attend 33 conversations", "fp16", 40, 40, 33, 2000, 16, group=32),
        # four draft tokens verified per sequence under a sliding window, some slots of the batch empty
        _attend("attend drafts window", "fp16", 32, 8, 16, 7000, 32, q_len=4, window=4096, idle=2),
        # a serving batch of long conversations, one scale for a whole head
        _attend("attend 128 long", "bf16", 64, 8, 128, 9216, 64, group=128),
        # one token of one sequence, stored and read back: latency
        _store("store 1", "bf16", 32, 8, 1, 1, 16, rope_dim=128),
        # a decode step of a batch at scattered positions, half of each head rotated, pairs side by side
        _store("store 200 partial", "fp16", 64, 8, 200, 1, 64, rope_dim=64, interleaved=True),
        # chunks of prompts
        _store("store chunks", "bf16", 64, 8, 16, 1023, 64, rope_dim=128),
        # a short conversation brought back to 16 bits
        _read("read 1 short", "bf16", 32, 8, 1, 333, 16),
        # sequences brought back to 16 bits, to become the prefix of others or to leave the machine
        _read("read 16 long", "fp16", 64, 8, 16, 8191, 64, group=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["attend", "attend", "store", "read"])
    most = [work(c) for c in listed() if c["op"] == op]
    while True:
        heads, kv_heads = rng.choice([(32, 32), (32, 8), (40, 40), (64, 8), (16, 2), (8, 1), (28, 4)])
        head_dim = rng.choice([128, 128, 128, 64, 256])
        group = rng.choice([g for g in (32, 64, 64, 128) if g <= head_dim])
        dtype, page = rng.choice(["bf16", "fp16"]), rng.choice([16, 32, 48, 64, 128])
        seqs = _log(rng, 1, 256)
        if op == "attend":
            q_len = rng.choice([1, 1, 1, 2, 3, 5, 8])
            window = rng.choice([0, 0, 0, _log(rng, 64, 8192) | 1])
            idle = rng.choice([0, 0, 1]) if seqs > 2 else 0
            c = _attend("", dtype, heads, kv_heads, seqs, q_len + (_log(rng, 1, 131072) | 1), page, group, head_dim, q_len, window, idle)
        else:
            chunk = 1 if rng.random() < 0.4 else _log(rng, 2, 8192) | 1
            rope = rng.choice([0, head_dim // 2, head_dim, head_dim]) if op == "store" else 0
            c = _tokens("", op, dtype, heads, kv_heads, seqs, chunk, page, group, head_dim, rope, rng.random() < 0.3, rng.random() < 0.7)
        c.pop("name")
        w = work(c)
        if w["bytes"] <= max(m["bytes"] for m in most) and w["flops"] <= max(m["flops"] for m in most) and _plain_bytes(c) <= 24e9:
            return c


def _plain_bytes(c):
    """What the plain attention holds at once, about: its scores and its copies of keys and values in 32 bits."""
    if c["op"] != "attend":
        return 0
    keys = c["keys"] + c["page"]
    return 4 * c["seqs"] * keys * (3 * c["q_len"] * c["heads"] + 4 * c["kv_heads"] * c["head_dim"])


def _lengths(c):
    """Lengths of the sequences, between a quarter of the longest and the longest; the last ``idle`` slots are empty."""
    got = []
    for b in range(c["seqs"]):
        f = 1.0 if b == 0 else 0.25 + 0.75 * ((b * 0.6180339887) % 1.0)
        got.append(max(c["q_len"], int(round(c["keys"] * f))) if b < c["seqs"] - c["idle"] else 0)
    return got


def _token_bytes(c):
    """Bytes of one token's key and value of one head as they are held."""
    return c["head_dim"] + 8 * (c["head_dim"] // c["group"])


def work(c):
    d, held = c["head_dim"], c["kv_heads"] * _token_bytes(c)
    t = c["seqs"] * c.get("chunk", 0)
    if c["op"] == "store":  # queries in and out; keys and values in, into the pages, and out again
        return {"bytes": t * (4 * c["heads"] * d + 8 * c["kv_heads"] * d + 2 * held + 4 * c["rope_dim"] + 8),
                "flops": t * (3 * (c["heads"] + c["kv_heads"]) * c["rope_dim"] + 2 * c["kv_heads"] * 8 * d)}
    if c["op"] == "read":
        return {"bytes": t * (4 * c["kv_heads"] * d + held + 8), "flops": 4 * t * c["kv_heads"] * d}
    keys, pairs, rows = 0, 0, 0
    for n in _lengths(c):
        if n == 0:
            continue
        keys += n - (max(0, n - c["q_len"] + 1 - c["window"]) if c["window"] else 0)
        pairs += sum(min(n - c["q_len"] + 1 + i, c["window"] or n) for i in range(c["q_len"]))
        rows += c["q_len"]
    return {"bytes": keys * held + c["seqs"] * c["q_len"] * c["heads"] * (4 * d + 4), "flops": 4 * d * c["heads"] * pairs}


# ---- the inputs -------------------------------------------------------------------------------------------------------------
class State:
    pass


def _randn(gen, shape, dtype, std=1.0):
    x = torch.empty(shape, dtype=dtype, device=DEV)
    return x.normal_(0.0, std, generator=gen)


def _rope_table(positions, rope_dim):
    """Cosines, then sines, of position * 10000^(-2 i / rope_dim), computed in 64 bits and kept in 32."""
    i = torch.arange(rope_dim // 2, dtype=torch.float64, device=DEV)
    angle = torch.arange(positions, dtype=torch.float64, device=DEV)[:, None] * 10000.0 ** (-2.0 * i / rope_dim)
    return torch.cat([angle.cos(), angle.sin()], 1).float()


def _pool(gen, c, n_pages):
    """Pages full of tokens: keys and values of unit variance with a few large channels, in 4 bits."""
    d, groups = c["head_dim"], c["head_dim"] // c["group"]
    pages = torch.empty(n_pages, c["kv_heads"], c["page"] * _token_bytes(c), dtype=torch.uint8, device=DEV)
    std = torch.ones(2, c["kv_heads"], 1, 1, d, device=DEV)
    std[0].view(c["kv_heads"], d)[:, :: d // 4] = 4.0
    step = max(1, 2 ** 25 // (2 * c["kv_heads"] * c["page"] * d))
    slot = torch.arange(16, device=DEV)
    for a in range(0, n_pages, step):
        n = min(step, n_pages - a)
        x = (_randn(gen, (n, 2, c["kv_heads"], c["page"] // 16, 16, d), torch.float32) * std).to(DTYPES[c["dtype"]])
        code, meta = _quantised(x, c["group"])
        rows = [_packed(code[:, i], _order(d, i)[slot % 4]) for i in range(2)]
        parts = rows + [meta[:, i].contiguous().view(torch.uint8).view(*rows[0].shape[:-1], 4 * groups) for i in range(2)]
        pages[a:a + n] = torch.cat([p.flatten(3) for p in parts], 3).flatten(2)
    return pages


def prepare(case, seed):
    c, s = case, State()
    s.case = c
    gen = torch.Generator(device=DEV).manual_seed(seed)
    if c["op"] == "attend":
        _prepare_attend(c, s, gen, seed)
    else:
        _prepare_tokens(c, s, gen)
    return s


def _prepare_attend(c, s, gen, seed):
    page, dt, lens = c["page"], DTYPES[c["dtype"]], _lengths(c)
    order = torch.randperm(c["seqs"], generator=torch.Generator().manual_seed(seed)).tolist()
    lens = [lens[j] for j in order]
    need = [-(-n // page) for n in lens]
    # pages of the pool are handed out in a shuffled order
    ids = torch.randperm(sum(need), generator=gen, device=DEV).to(torch.int32)
    s.pages = _pool(gen, c, sum(need))
    s.table = torch.zeros(c["seqs"], max(need), dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(need):
        s.table[b, :n] = ids[at:at + n]
        at += n
    s.seq_len = torch.tensor(lens, dtype=torch.int32, device=DEV)
    # scores of trained models spread over several units: queries longer than unit variance
    s.q = _randn(gen, (c["seqs"], c["q_len"], c["heads"], c["head_dim"]), dt, 2.0)
    s.out = torch.empty_like(s.q)
    s.lse = torch.empty(c["seqs"], c["q_len"], c["heads"], dtype=torch.float32, device=DEV)
    if own:
        from paper_2609_03079_b200 import binding as ls
        s.kv = ls.ls_paged_kv4_create(s.pages, c["heads"], c["head_dim"], c["page"], dtype=dt, group=c["group"], max_seqs=c["seqs"], max_q_len=c["q_len"])


def _prepare_tokens(c, s, gen):
    page, dt, T = c["page"], DTYPES[c["dtype"]], c["seqs"] * c["chunk"]
    limit = max(32768, 2 * c["chunk"])
    start = torch.randint(0, limit - c["chunk"], (c["seqs"],), generator=gen, device=DEV)
    per = -(-c["chunk"] // page) + 1
    ids = torch.randperm(c["seqs"] * per, generator=gen, device=DEV).to(torch.int32).view(c["seqs"], per)
    s.table = torch.zeros(c["seqs"], -(-limit // page) + 1, dtype=torch.int32, device=DEV)
    s.table.scatter_(1, torch.div(start[:, None], page, rounding_mode="floor") + torch.arange(per, device=DEV), ids)
    s.seq = torch.arange(c["seqs"], device=DEV, dtype=torch.int32).repeat_interleave(c["chunk"])
    s.pos = (start[:, None] + torch.arange(c["chunk"], device=DEV)).reshape(-1).to(torch.int32)
    s.pages = _pool(gen, c, c["seqs"] * per)
    h, g, d = c["heads"], c["kv_heads"], c["head_dim"]
    s.k_out, s.v_out = (torch.empty(T, g, d, dtype=dt, device=DEV) for _ in range(2))
    s.rope = _rope_table(limit, c["rope_dim"]) if c["rope_dim"] else None
    if c["op"] == "store":
        if c["fused"]:  # slices of one projection's output
            s.q, s.k, s.v = _randn(gen, (T, h + 2 * g, d), dt).split([h, g, g], 1)
        else:
            s.q, s.k, s.v = (_randn(gen, (T, n, d), dt) for n in (h, g, g))
        s.q_out = torch.empty(T, h, d, dtype=dt, device=DEV)
    if own:
        from paper_2609_03079_b200 import binding as ls
        s.kv = ls.ls_paged_kv4_create(s.pages, h, d, page, dtype=dt, group=c["group"], rope=s.rope, rope_interleaved=c["interleaved"])


# ---- one pass ---------------------------------------------------------------------------------------------------------------
def run(s):
    c = s.case
    if not own:
        return {"attend": _plain_attend, "store": _plain_store, "read": _plain_read}[c["op"]](s)
    from paper_2609_03079_b200 import binding as ls
    if c["op"] == "attend":
        ls.ls_paged_kv4_attend(s.kv, s.q, s.out, s.seq_len, s.table, window=c["window"], lse=s.lse)
        return s.out, s.lse
    if c["op"] == "read":
        ls.ls_paged_kv4_read(s.kv, s.k_out, s.v_out, s.seq, s.pos, s.table)
        return s.k_out, s.v_out
    # what the pages hold of the tokens is returned as the values that it stands for
    ls.ls_paged_kv4_append(s.kv, s.q, s.k, s.v, s.q_out, s.seq, s.pos, s.table)
    ls.ls_paged_kv4_read(s.kv, s.k_out, s.v_out, s.seq, s.pos, s.table)
    return s.q_out, s.k_out, s.v_out


def _order(d, value):
    """[4, d]: the component at each place of a code row (eight to a word of four bytes, the lowest bits first), by the row's
    number modulo 4."""
    place, row = torch.arange(d, device=DEV), torch.arange(4, device=DEV)[:, None]
    word, i = place // 8, place % 8
    if value:  # pieces of eight words trade places; a word has four components of one half of 64 and four of the other
        n = d // 64
        at = (word // 8 ^ (row % n if n == 4 else row // 2 % n)) * 8 + word % 8
        return at % n * 64 + i // 4 * 32 + at // n * 4 + i % 4
    n = min(4, d // 32)  # words that four threads take turns at; halves trade places where there are two
    half = word // (4 * n) ^ (row % 2 if d == 256 else row * 0)
    return ((half * n + word % n) * 4 + word // n % 4) * 8 + i


def _quantised(x, group):
    """Codes (uint8, of x's shape) and [..., groups, 2] scales and zeros of x's type."""
    y = x.float().unflatten(-1, (-1, group))
    zero = y.amin(-1, keepdim=True)
    scale = ((y.amax(-1, keepdim=True) - zero) / 15.0).to(x.dtype)
    code = torch.where(scale > 0, torch.round((y - zero) / scale.float()), 0.0).clamp_(max=15.0)
    return code.to(torch.uint8).flatten(-2), torch.cat([scale, zero.to(x.dtype)], -1)


def _packed(code, order):
    """Two codes to a byte; order [rows, d] for code [..., rows, d]."""
    code = code.gather(-1, order.expand(code.shape))
    return code[..., 0::2] | code[..., 1::2] << 4


def _values(rows, meta, order, group):
    """Fp32 components of code rows [..., rows, d / 2] with meta [..., rows, groups, 2]."""
    code = torch.stack([rows & 15, rows >> 4], -1).flatten(-2).float()
    x = torch.empty_like(code).scatter_(-1, order.expand(code.shape), code).unflatten(-1, (-1, group))
    return (x * meta[..., :1].float() + meta[..., 1:].float()).flatten(-2)


def _places(s):
    """Page and head of every token, byte offsets of its two code rows and its two rows of scales and zeros, and its row's number."""
    c, page, d = s.case, s.case["page"], s.case["head_dim"]
    pos = s.pos.long()
    at = s.table[s.seq.long(), torch.div(pos, page, rounding_mode="floor")].long()
    slot, m = pos % page, 4 * d // c["group"]
    tile, row = torch.div(slot, 16, rounding_mode="floor") * (16 * _token_bytes(c)), slot % 16
    first = [tile + row * (d // 2), tile + (16 + row) * (d // 2), tile + 16 * d + row * m, tile + 16 * d + (16 + row) * m]
    offsets = [f[:, None, None] + torch.arange(n, device=DEV) for f, n in zip(first, (d // 2, d // 2, m, m))]
    return at[:, None, None], torch.arange(c["kv_heads"], device=DEV)[:, None], offsets, row


def _plain_read(s):
    c, dt = s.case, s.k_out.dtype
    page, head, offsets, row = _places(s)
    for i, out in enumerate((s.k_out, s.v_out)):
        meta = s.pages[page, head, offsets[2 + i]].view(dt).unflatten(-1, (-1, 2))
        out.copy_(_values(s.pages[page, head, offsets[i]], meta, _order(c["head_dim"], i)[row % 4][:, None], c["group"]))
    return s.k_out, s.v_out


def _rotated(s, x):
    r = s.case["rope_dim"]
    if r == 0:
        return x
    cos, sin = s.rope[s.pos.long()].to(x.dtype).view(-1, 1, 2, r // 2).unbind(2)
    a, b = (x[..., 0:r:2], x[..., 1:r:2]) if s.case["interleaved"] else (x[..., : r // 2], x[..., r // 2:r])
    y = (a * cos - b * sin, b * cos + a * sin)
    y = torch.stack(y, -1).flatten(-2) if s.case["interleaved"] else torch.cat(y, -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_store(s):
    c, dt = s.case, s.k.dtype
    page, head, offsets, row = _places(s)
    for i, x in enumerate((_rotated(s, s.k.double()).float().to(dt), s.v)):
        code, meta = _quantised(x, c["group"])
        s.pages[page, head, offsets[i]] = _packed(code, _order(c["head_dim"], i)[row % 4][:, None])
        s.pages[page, head, offsets[2 + i]] = meta.contiguous().view(torch.uint8).flatten(-2)
    s.q_out.copy_(_rotated(s, s.q.float()))
    return (s.q_out,) + _plain_read(s)


def _plain_attend(s):
    c, d, G = s.case, s.case["head_dim"], s.case["group"]
    B, n, H, _ = s.q.shape
    hk, groups, row = c["kv_heads"], d // G, torch.arange(16, device=DEV)
    tiles = s.pages[s.table.long()].unflatten(-1, (-1, 16 * _token_bytes(c))).transpose(2, 3).flatten(1, 2)  # [seqs, tiles, kv_heads, bytes]
    rows = tiles[..., : 16 * d].unflatten(-1, (2, 16, d // 2))
    meta = tiles[..., 16 * d:].contiguous().view(s.q.dtype).unflatten(-1, (2, 16, groups, 2))
    k, v = (_values(rows[:, :, :, i], meta[:, :, :, i], _order(d, i)[row % 4], G).transpose(2, 3).flatten(1, 2) for i in range(2))  # [seqs, keys, kv_heads, d]
    q = s.q.float().view(B, n, hk, H // hk, d)
    at = torch.arange(k.shape[1], device=DEV)
    pos = s.seq_len[:, None] - n + torch.arange(n, device=DEV)
    seen = at <= pos[..., None]
    if c["window"]:
        seen &= at > pos[..., None] - c["window"]
    score = torch.where(seen[:, :, None, None], torch.einsum("bnhgd,bkhd->bnhgk", q, k) * d ** -0.5, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    e = torch.exp(score.sub_(top))
    total = e.sum(-1, keepdim=True)
    out = torch.where(total > 0, torch.einsum("bnhgk,bkhd->bnhgd", e, v) / total, 0.0)
    lse = top + torch.log(total)
    return out.reshape(B, n, H, d).to(s.q.dtype), lse.reshape(B, n, H)


# ---- the definitions in 64 bits ---------------------------------------------------------------------------------------------
def exact(case, seed):
    c, s = case, prepare(case, seed)
    return {"attend": _exact_attend, "store": _exact_store, "read": _exact_read}[c["op"]](c, s)


def _nibble(c, value, row):
    """Byte and shift of every component in code row ``row`` (a tensor; the result has one more dimension)."""
    d = c["head_dim"]
    x, row = torch.arange(d, device=DEV), row[..., None]
    if value:
        n = d // 64
        word = x % 32 // 4 * n + x // 64
        swap = {1: row * 0, 2: row // 2 % 2, 4: row % 4}[n]
        word = (word // 8 ^ swap) * 8 + word % 8
        i = x % 64 // 32 * 4 + x % 4
    else:
        n = min(4, d // 32)
        turn, lane = x // 32, x // 8 % 4
        half = turn // n ^ (row % 2 if d == 256 else row * 0)
        word = half * 4 * n + lane * n + turn % n
        i = (x % 8).expand(word.shape)
    return word * 4 + i.expand(word.shape) // 2, i.expand(word.shape) % 2 * 4


def _held(c, blocks, slot):
    """Keys and values (64 bits) held in slots ``slot`` [t] of blocks [t, kv_heads, bytes]."""
    d, groups = c["head_dim"], c["head_dim"] // c["group"]
    tile, row = torch.div(slot, 16, rounding_mode="floor") * (16 * _token_bytes(c)), slot % 16
    both = []
    for value in (0, 1):
        byte, shift = _nibble(c, value, row)
        byte = byte + (tile + (16 * value + row) * (d // 2))[:, None]
        code = blocks.gather(2, byte[:, None].expand(-1, blocks.shape[1], -1)).long() >> shift[:, None] & 15
        at = (tile + 16 * d + (16 * value + row) * 4 * groups)[:, None] + torch.arange(4 * groups, device=DEV)
        meta = blocks.gather(2, at[:, None].expand(-1, blocks.shape[1], -1)).contiguous().view(DTYPES[c["dtype"]]).double()
        scale, zero = (meta[..., k::2].repeat_interleave(c["group"], -1) for k in (0, 1))
        both.append(code.double() * scale + zero)
    return both


def _exact_read(c, s):
    pos, out = s.pos.long(), []
    at = s.table[s.seq.long(), torch.div(pos, c["page"], rounding_mode="floor")].long()
    for a in range(0, pos.numel(), 4096):
        out.append(_held(c, s.pages[at[a:a + 4096]], pos[a:a + 4096] % c["page"]))
    return tuple(torch.cat(t) for t in zip(*out))


def _exact_store(c, s):
    """Rotation as a product of complex numbers, codes as the nearest of the sixteen levels."""
    r, dt = c["rope_dim"], DTYPES[c["dtype"]]

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

    def held(x):
        y = x.to(dt).double().reshape(*x.shape[:-1], -1, c["group"])
        low, high = y.min(-1, keepdim=True).values, y.max(-1, keepdim=True).values
        scale = ((high - low) / 15).to(dt).double()
        level = (y - low) / torch.where(scale > 0, scale, 1.0)
        below = level.floor()
        over = level - below
        level = below + ((over > 0.5) | ((over == 0.5) & (below % 2 == 1)))
        return (low + level.clamp(max=15) * scale).reshape(x.shape)

    return turned(s.q), held(turned(s.k)), held(s.v.double())


def _exact_attend(c, s):
    """Sequence by sequence, one softmax over what each token sees."""
    B, n, H, D = s.q.shape
    page = c["page"]
    out = torch.zeros(B, n, H, D, dtype=torch.float64, device=DEV)
    lse = torch.full((B, n, H), -math.inf, dtype=torch.float64, device=DEV)
    for b, length in enumerate(s.seq_len.tolist()):
        if length == 0:
            continue
        parts = []
        for a in range(0, length, 64 * page):
            at = torch.arange(a, min(length, a + 64 * page), device=DEV)
            parts.append(_held(c, s.pages[s.table[b, torch.div(at, page, rounding_mode="floor")].long()], at % page))
        k, v = (torch.cat(t).transpose(0, 1) for t in zip(*parts))  # [kv_heads, length, D]
        for i in range(n):
            end = length - n + i + 1
            begin = max(0, end - c["window"]) if c["window"] else 0
            score = s.q[b, i].double().view(c["kv_heads"], -1, D) @ k[:, begin:end].transpose(1, 2) / math.sqrt(D)
            lse[b, i] = torch.logsumexp(score, -1).view(-1)
            out[b, i] = (torch.softmax(score, -1) @ v[:, begin:end]).view(H, D)
    return out, lse
