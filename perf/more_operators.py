"""The operators of attention over a key/value cache held in 4 bits, as a model's forward pass calls them: what is timed, and
what the results must be.

  rope      queries and keys of each head: root-mean-square norm, rotation by position, optionally a Hadamard rotation
  append    new keys and values into the cache, with the values that the codes stand for
  attention softmax(scale q k^T) v over the cache: one token a sequence, a few, or a chunk of a prompt
  weights   the probability that each cached token received, summed over queries and heads of a group, added up
  evict     the tokens with the most accumulated weight, and the most recent ones, stay in the cache

Cache: pages [page][kv head][bytes] of page_size tokens, in groups of 16: key codes [token][D / 2], key parameters
[token][scale, offset] in bf16, then the same of the values.  Two codes a byte, the even one in the low half; value =
offset + scale * code.  A table
[sequence][page of the sequence] says which pages hold a sequence, `lengths` how many tokens (slots) it has.  The n queries
of a sequence are its last n tokens: query i sees the slots below length - n + i + 1.
"""
import math

import torch

own = False

FLOAT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one decoded token's queries and keys: launch latency
        dict(name="rope_token", op="rope", tokens=1, q_heads=32, heads=8, dim=128, rot=128, dtype="bf16", pairs="halves", hadamard=True),
        # a calibration set through a 70B-size layer with grouped queries: views of one fused projection's output
        dict(name="rope_prompt", op="rope", tokens=16384, q_heads=64, heads=8, dim=128, rot=128, dtype="bf16", pairs="halves", hadamard=True),
        # sixteen sequences decode one token each
        dict(name="append_token", op="append", batch=16, queries=1, length=2048, heads=8, dim=128, page=64, dtype="bf16"),
        # ragged prompts of a 13B-size model (40 heads, no groups)
        dict(name="append_prompts", op="append", batch=12, queries=2048, length=4096, heads=40, dim=128, page=16, dtype="fp16"),
        # one sequence decodes one token after a short prompt: latency
        dict(name="attention_token", op="attention", batch=1, queries=1, length=1024, q_heads=32, heads=8, dim=128, page=64, dtype="bf16"),
        # one very long sequence, 70B-size heads: the long axis is split
        dict(name="attention_long", op="attention", batch=1, queries=1, length=131072, q_heads=64, heads=8, dim=128, page=128, dtype="bf16"),
        # a serving batch of ragged sequences
        dict(name="attention_batch", op="attention", batch=64, queries=1, length=16384, q_heads=32, heads=8, dim=128, page=64, dtype="bf16"),
        # the last chunk of a long prompt
        dict(name="attention_chunk", op="attention", batch=1, queries=4096, length=16384, q_heads=32, heads=8, dim=128, page=64, dtype="bf16"),
        # the weights of a decoding batch's tokens
        dict(name="weights_batch", op="weights", batch=16, queries=1, length=8192, q_heads=32, heads=8, dim=128, page=64, dtype="bf16"),
        # the weights after a chunk of a prompt, odd sizes, narrow heads
        dict(name="weights_chunk", op="weights", batch=2, queries=777, length=8191, q_heads=16, heads=4, dim=64, page=32, dtype="fp16"),
        # one sequence passes its budget by a few tokens
        dict(name="evict_one", op="evict", batch=1, length=2056, keep=2048, recent=256, heads=8, dim=128, page=64),
        # a serving batch is cut to its budget
        dict(name="evict_batch", op="evict", batch=32, length=16384, keep=4096, recent=512, heads=8, dim=128, page=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["rope", "append", "attention", "attention", "weights", "evict"])
    dim = rng.choice([64, 128, 128, 256])
    heads = rng.choice([1, 2, 4, 8, 8, 16, 32])
    page = rng.choice([16, 32, 64, 128, 256])
    dtype = rng.choice(["bf16", "fp16"])
    if op == "rope":
        dim = rng.choice([64, 80, 96, 128, 128, 256])
        q_heads = heads * rng.choice([1, 2, 4, 8])
        tokens = min(_log_uniform(rng, 1, 16384), 150000000 // ((q_heads + heads) * dim))
        rot = dim if rng.random() < 0.7 else dim // 32 * 16
        return dict(op=op, tokens=tokens, q_heads=q_heads, heads=heads, dim=dim, rot=rot, dtype=rng.choice(["bf16", "fp16", "fp32"]),
                    pairs=rng.choice(["halves", "neighbours"]), hadamard=dim in (64, 128, 256) and rng.random() < 0.5)
    if op == "append":
        batch, queries = _log_uniform(rng, 1, 64), 1 if rng.random() < 0.3 else _log_uniform(rng, 1, 4096)
        queries = max(1, min(queries, 100000000 // (batch * heads * dim)))
        return dict(op=op, batch=batch, queries=queries, length=queries + _log_uniform(rng, 1, 2048), heads=heads, dim=dim, page=page,
                    dtype=rng.choice(["bf16", "fp16", "fp32"]))
    if op == "evict":
        batch = _log_uniform(rng, 1, 32)
        length = max(2, min(_log_uniform(rng, 2, 32768), 500000000 // (batch * heads * dim)))
        keep = max(1, int(length * rng.uniform(0.1, 1)))
        return dict(op=op, batch=batch, length=length, keep=keep, recent=int(keep * rng.uniform(0, 0.5)), heads=heads, dim=dim, page=page)
    group = rng.choice([1, 2, 4, 8, 8, 5]) if heads <= 16 else 1
    kind = rng.random()
    queries = 1 if kind < 0.5 else rng.randint(2, 9) if kind < 0.7 else _log_uniform(rng, 16, 2048)
    batch = _log_uniform(rng, 1, 64 if queries < 16 else 4)
    # the cache's values, and the products of queries and keys that the plain form holds
    most = min(600000000 // (batch * heads * dim), 500000000 // (batch * heads * group * queries))
    length = max(queries, min(_log_uniform(rng, 16, 131072), most))
    return dict(op=op, batch=batch, queries=queries, length=length, q_heads=heads * group, heads=heads, dim=dim, page=page, dtype=dtype)


def _spread(count, most):
    """Ragged sizes from about a quarter of `most` to all of it, the first one all of it."""
    return [max(1, int(most * (1 - 0.75 * (i * 0.6180339887 % 1)))) for i in range(count)]


def _sizes(case):
    """(queries of each sequence, tokens of each sequence)"""
    queries = _spread(case["batch"], case.get("queries", 1))
    return queries, [max(q, n) for q, n in zip(queries, _spread(case["batch"], case["length"]))]


def work(case):
    dim, heads = case["dim"], case["heads"]
    if case["op"] == "rope":
        n = case["tokens"] * (case["q_heads"] + heads) * dim
        return {"bytes": 2 * n * FLOAT[case["dtype"]].itemsize + 4 * case["tokens"], "flops": n * (10 + case["hadamard"] * math.log2(dim))}
    queries, lengths = _sizes(case)
    if case["op"] == "append":  # keys and values read, codes, parameters and values written
        size = FLOAT[case["dtype"]].itemsize
        return {"bytes": sum(queries) * heads * (4 * dim * size + dim + 8), "flops": sum(queries) * heads * 2 * dim * 8}
    if case["op"] == "evict":  # weights and positions read, those that stay written, about keep / n of the rest moved
        kept = [min(n, case["keep"]) for n in lengths]
        moved = sum(k * (n - k) // n for n, k in zip(lengths, kept))
        return {"bytes": heads * (8 * sum(lengths) + 8 * sum(kept) + 2 * moved * (dim + 8)), "flops": heads * sum(lengths)}
    pairs = sum(q * n - q * (q - 1) // 2 for q, n in zip(queries, lengths)) * case["q_heads"]
    rows = sum(queries) * case["q_heads"]
    if case["op"] == "weights":  # queries, their sums, keys; weights read and written
        return {"bytes": sum(lengths) * heads * (dim // 2 + 12) + rows * (2 * dim + 4), "flops": 2 * dim * pairs}
    return {"bytes": sum(lengths) * heads * (dim + 8) + rows * (4 * dim + 4), "flops": 4 * dim * pairs}


# ------------------------------------------------------------------------------------------------ plain forms
def _hadamard(dim, device):
    i = torch.arange(dim, device=device)
    ones = ((i[:, None] & i[None, :])[..., None] >> torch.arange(8, device=device)) & 1
    return (1 - 2 * (ones.sum(-1) % 2)).float() / math.sqrt(dim)


def _rope(x, gamma, cos, sin, pairs, hadamard):
    """x [tokens][heads][dim] in its type; cos, sin [tokens][rot / 2] in fp32."""
    h = x.float()
    h = h * torch.rsqrt(torch.mean(h * h, -1, keepdim=True) + EPS) * gamma.float()
    half, cos, sin = cos.shape[-1], cos[:, None], sin[:, None]
    r = h[..., :2 * half]
    if pairs == "halves":
        a, b = r[..., :half], r[..., half:]
        r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
    else:
        a, b = r[..., 0::2], r[..., 1::2]
        r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
    h = torch.cat((r, h[..., 2 * half:]), -1)
    return (torch.matmul(h, _hadamard(h.shape[-1], h.device)) if hadamard else h).to(x.dtype)


def _bf16_bits_down(v):
    """The largest bf16 value not above v (finite fp32), in fp32."""
    bits = v.contiguous().view(torch.int32)
    cut = bits & -65536
    return torch.where((bits < 0) & (cut != bits), cut + 65536, cut).view(torch.float32)


def _quantize(x):
    """(codes, scale, offset) of x [..., dim] in fp32; scale and offset [..., 1] are bf16 values."""
    off = _bf16_bits_down(x.amin(-1, keepdim=True) + 0.0)
    fifteen = x.new_full((), 15.0)  # (a tensor: by a plain number torch multiplies with the reciprocal)
    scale = -_bf16_bits_down(-((x.amax(-1, keepdim=True) - off) / fifteen))
    codes = torch.round((x - off) / torch.where(scale > 0, scale, 1.0))
    return torch.where(scale > 0, codes, 0.0), scale, off


def _packed(codes, scale, off):
    """Codes [..., dim / 2] and parameters [..., 4] in bytes."""
    c = codes.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4), torch.cat((scale, off), -1).to(torch.bfloat16).contiguous().view(torch.uint8)


GROUP = 16  # tokens whose codes and parameters lie together


def _parts(pages, dim):
    """Views of the key codes, key parameters, value codes and value parameters: [page][head][group][token][bytes]."""
    groups = pages.unflatten(-1, (-1, GROUP * (dim + 8)))
    kc, kp, vc, vp = groups.split([GROUP * b for b in (dim // 2, 4, dim // 2, 4)], -1)
    return tuple(v.unflatten(-1, (GROUP, -1)) for v in (kc, kp, vc, vp))


def _values(codes, params, table, most):
    """Values in fp32 [sequence][head][slot < most][dim] of all pages' codes and parameters."""
    at = table[:, :-(-most // (codes.shape[2] * GROUP))].long().clamp(min=0)
    c, p = codes[at], params[at].contiguous().view(torch.bfloat16).float()
    c = torch.stack((c & 15, c >> 4), -1).flatten(-2).float()
    v = p[..., 1:] + p[..., :1] * c
    return v.transpose(1, 2).flatten(2, 4)[:, :, :most]


def _padded(s):
    """(row of Q of each sequence's query i, whether there is one): [sequence][queries at most]"""
    i = torch.arange(s["most_queries"], device="cuda")
    n = (s["starts"][1:] - s["starts"][:-1])[:, None]
    return torch.where(i < n, s["starts"][:-1, None] + i, 0).long(), i < n


def _logits(s):
    """(q k^T scale [sequence][head][query x group][slot], -inf where masked, rows, there)"""
    rows, there = _padded(s)
    group, batch = s["q_heads"] // s["heads"], rows.shape[0]
    kc, kp, _, _ = _parts(s["pages"], s["dim"])
    k = _values(kc, kp, s["table"], s["most"])
    q = s["q"][rows].float().unflatten(2, (s["heads"], group)).permute(0, 2, 1, 3, 4).flatten(2, 3)
    logits = torch.matmul(q, k.transpose(-1, -2)) * s["scale"]
    n = (s["starts"][1:] - s["starts"][:-1])[:, None]
    sees = s["lengths"][:, None] - n + torch.arange(rows.shape[1], device="cuda") + 1
    sees = torch.where(there, sees, 0).repeat_interleave(group, 1)[:, None, :, None]
    return torch.where(torch.arange(s["most"], device="cuda") < sees, logits, -math.inf), rows, there


def _back(x, rows, there, s, into):
    """x [sequence][head][query x group][...] to the rows of Q: into [token][query head][...]"""
    group = s["q_heads"] // s["heads"]
    x = x.unflatten(2, (rows.shape[1], group)).transpose(1, 2).flatten(2, 3)
    into[rows[there]] = x[there].to(into.dtype)
    return into


def _attention(s):
    logits, rows, there = _logits(s)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
    total = p.sum(-1, keepdim=True)
    _, _, vc, vp = _parts(s["pages"], s["dim"])
    v = _values(vc, vp, s["table"], s["most"])
    used = torch.arange(s["most"], device="cuda")[:, None] < s["lengths"][:, None, None, None]
    o = torch.matmul(p, torch.where(used, v, 0.0)) / torch.where(total > 0, total, 1.0)
    lse = (top + torch.log(total))[..., 0]
    return (_back(o, rows, there, s, torch.empty_like(s["q"])),
            _back(lse, rows, there, s, torch.empty(s["q"].shape[:2], device="cuda")))


def _weights(s):
    logits, rows, there = _logits(s)
    group = s["q_heads"] // s["heads"]
    lse = s["lse"][rows].unflatten(2, (s["heads"], group)).permute(0, 2, 1, 3).flatten(2, 3)[..., None]
    got = torch.where(logits > -math.inf, torch.exp(logits - lse), 0.0).sum(2)
    slot = torch.arange(s["most"], device="cuda")
    n = (s["starts"][1:] - s["starts"][:-1])[:, None, None]
    old = torch.where(slot < s["lengths"][:, None, None] - n, s["weights"][..., :s["most"]], 0.0)
    out = s["weights_out"]
    out[..., :s["most"]] = torch.where(slot < s["lengths"][:, None, None], old + got, out[..., :s["most"]])
    return out


def _slots(s):
    """(sequence of each new token, its slot)"""
    n = s["starts"][1:] - s["starts"][:-1]
    seq = torch.repeat_interleave(torch.arange(n.shape[0], device="cuda"), n.long(), output_size=s["k"].shape[0])
    return seq, (s["lengths"] - s["starts"][1:])[seq] + torch.arange(seq.shape[0], device="cuda")


def _append(s):
    seq, slot = _slots(s)
    page, at = s["table"][seq, slot // s["page"]].long(), (slot % s["page"]).long()
    group, at = at // GROUP, at % GROUP
    kc, kp, vc, vp = _parts(s["pages"], s["dim"])
    k, v = _quantize(s["k"].float()), _quantize(s["v"].float())
    kc[page, :, group, at], kp[page, :, group, at] = _packed(*k)
    vc[page, :, group, at], vp[page, :, group, at] = _packed(*v)
    return {"pages": s["pages"], "keys": (k[2] + k[1] * k[0]).to(s["k"].dtype), "values": (v[2] + v[1] * v[0]).to(s["v"].dtype)}


def _evict(s):
    most, keep = s["most"], s["keep"]
    slot = torch.arange(most, device="cuda")
    used = (slot < s["lengths"][:, None, None]).expand(-1, s["heads"], -1)
    w, pos = s["weights"][..., :most], s["positions"][..., :most]
    newest = torch.where(used, pos, -1).amax(-1, keepdim=True)
    key = torch.where(pos > newest - s["recent"], math.inf, w)
    order = torch.sort(torch.where(used, key, -math.inf), dim=-1, descending=True, stable=True).indices
    rank = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order).contiguous())
    stays = used & (rank < keep)
    hole, mover = (slot < keep) & used & ~stays, (slot >= keep) & stays
    # the i-th slot that moves goes to the i-th that is free
    free = torch.full((*w.shape[:2], most + 1), most, device="cuda")
    free.scatter_(-1, torch.where(hole, hole.cumsum(-1) - 1, most), slot.expand_as(order).contiguous())
    seq, head, src = torch.nonzero(mover, as_tuple=True)
    dst = free[seq, head, (mover.cumsum(-1) - 1)[seq, head, src]]
    p = s["page"]
    from_page, to_page = s["table"][seq, src // p].long(), s["table"][seq, dst // p].long()
    for part in _parts(s["pages"], s["dim"]):
        part[to_page, head, dst % p // GROUP, dst % GROUP] = part[from_page, head, src % p // GROUP, src % GROUP]
    still = stays & (slot < keep)
    w_out, p_out = s["weights_out"], s["positions_out"]
    w_out[..., :most] = torch.where(still, w, w_out[..., :most])
    p_out[..., :most] = torch.where(still, pos, p_out[..., :most])
    w_out[seq, head, dst], p_out[seq, head, dst] = w[seq, head, src], pos[seq, head, src]
    s["lengths_out"].copy_(s["lengths"].clamp(max=keep))
    return {"pages": s["pages"], "weights": w_out, "positions": p_out, "lengths": s["lengths_out"]}


# ------------------------------------------------------------------------------------------------ inputs
def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _cache(case, g, s):
    """Pages in no order, the cache filled with keys and values of a rotated model: no outlier channels, offsets by head."""
    queries, lengths = _sizes(case)
    dim, heads, page, batch = case["dim"], case["heads"], case["page"], case["batch"]
    s["most"], s["most_queries"] = max(lengths), max(queries)
    need = [-(-n // page) for n in lengths]
    count = sum(need) + 3
    order = torch.randperm(count, device="cuda", generator=g).int()
    table = torch.full((batch, max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    pages = torch.zeros(count, heads, page * (dim + 8), dtype=torch.uint8, device="cuda")
    kc, kp, vc, vp = _parts(pages, dim)
    step = max(1, (1 << 27) // (heads * page * dim))
    for a in range(0, count, step):
        shape = kc[a:a + step].shape[:4]
        mean = 0.5 * _normal(g, 1, heads, 1, 1, dim)
        kc[a:a + step], kp[a:a + step] = _packed(*_quantize(_normal(g, *shape, dim) + mean))
        vc[a:a + step], vp[a:a + step] = _packed(*_quantize(_normal(g, *shape, dim) * torch.exp(0.3 * _normal(g, *shape, 1))))
    s["pages"], s["table"], s["page"] = pages, table, page
    s["lengths"] = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    s["starts"] = torch.tensor([sum(queries[:b]) for b in range(batch + 1)], dtype=torch.int32, device="cuda")
    return sum(queries), table.shape[1] * page


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = dict(case)
    dim, heads = case["dim"], case["heads"]
    if case["op"] == "rope":
        tokens, q_heads, dtype = case["tokens"], case["q_heads"], FLOAT[case["dtype"]]
        # queries, keys and values of one projection; the positions of a long sequence's last tokens
        qkv = _normal(g, tokens, q_heads + 2 * heads, dim).to(dtype)
        s["q"], s["k"] = qkv[:, :q_heads], qkv[:, q_heads:q_heads + heads]
        s["positions"] = torch.arange(100000, 100000 + tokens, dtype=torch.int32, device="cuda")
        s["inv_freq"] = (500000.0 ** (-torch.arange(0, case["rot"], 2, device="cuda", dtype=torch.float64) / case["rot"])).float()
        s["q_gamma"], s["k_gamma"] = ((1 + 0.2 * _normal(g, dim)).to(dtype) for _ in range(2))
        s["q_out"] = torch.empty(tokens, q_heads, dim, dtype=dtype, device="cuda")
        s["k_out"] = torch.empty(tokens, heads, dim, dtype=dtype, device="cuda")
        return s
    total, slots = _cache(case, g, s)
    if case["op"] == "append":
        dtype = FLOAT[case["dtype"]]
        kv = (_normal(g, total, 2 * heads, dim) + 0.5 * _normal(g, 1, 2 * heads, dim)).to(dtype)
        s["k"], s["v"] = kv[:, :heads], kv[:, heads:]
        s["keys"], s["values"] = (torch.empty(total, heads, dim, dtype=dtype, device="cuda") for _ in range(2))
        return s
    if case["op"] == "evict":
        shape = (case["batch"], heads, slots)
        # a few tokens get most of the weight; slots are in no order of positions after earlier evictions
        s["weights"] = torch.empty(shape, device="cuda").exponential_(generator=g).pow_(3)
        s["positions"] = torch.argsort(torch.rand(shape, device="cuda", generator=g), -1).int()
        s["weights_out"], s["positions_out"] = torch.zeros_like(s["weights"]), torch.zeros_like(s["positions"])
        s["lengths_out"] = torch.zeros_like(s["lengths"])
        return s
    s["scale"] = 1 / math.sqrt(dim)
    s["q"] = (1.5 * _normal(g, total, case["q_heads"], dim)).to(FLOAT[case["dtype"]])
    if case["op"] == "weights":
        s["lse"] = _attention(s)[1]
        s["weights"] = torch.rand(case["batch"], heads, slots, device="cuda", generator=g)
        s["weights_out"] = torch.zeros_like(s["weights"])
    else:
        s["out"] = torch.empty_like(s["q"])
        s["sums"] = torch.empty(s["q"].shape[:2], device="cuda")
    return s


# ------------------------------------------------------------------------------------------------ one pass
def _run_plain(s):
    if s["op"] == "rope":
        angle = s["positions"].double()[:, None] * s["inv_freq"].double()
        cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
        return {"q": _rope(s["q"], s["q_gamma"], cos, sin, s["pairs"], s["hadamard"]),
                "k": _rope(s["k"], s["k_gamma"], cos, sin, s["pairs"], s["hadamard"])}
    if s["op"] == "append":
        return _append(s)
    if s["op"] == "evict":
        return _evict(s)
    if s["op"] == "weights":
        return _weights(s)
    o, lse = _attention(s)
    return {"out": o, "lse": lse}


def _run_own(s):
    import paper_2511_04063_b200 as dq

    if s["op"] == "rope":
        flags = dq.DQ_QK_NORM | (dq.DQ_QK_NEIGHBOURS if s["pairs"] == "neighbours" else 0) | (dq.DQ_QK_HADAMARD if s["hadamard"] else 0)
        dq.dq_qk_norm_rope(s["q"], s["k"], s["positions"], s["inv_freq"], s["q_out"], s["k_out"], q_gamma=s["q_gamma"],
                           k_gamma=s["k_gamma"], eps=EPS, flags=flags)
        return {"q": s["q_out"], "k": s["k_out"]}
    if "cache" not in s:  # a program's handle of its cache
        s["cache"] = dq.dq_kv_cache(s["pages"], s["table"], s["lengths"], s["dim"])
    if s["op"] == "append":
        dq.dq_kv_append(s["k"], s["v"], s["cache"], starts=s["starts"], k_values=s["keys"], v_values=s["values"])
        return {"pages": s["pages"], "keys": s["keys"], "values": s["values"]}
    if s["op"] == "weights":
        dq.dq_kv_attention_weights(s["q"], s["lse"], s["cache"], s["scale"], s["weights_out"], weights=s["weights"], starts=s["starts"])
        return s["weights_out"]
    if "workspace" not in s:
        size = dq.dq_kv_evict_workspace(s["batch"], s["heads"], s["keep"]) if s["op"] == "evict" else dq.dq_kv_attention_workspace(s["dim"])
        s["workspace"] = torch.zeros(size, dtype=torch.uint8, device="cuda")
    if s["op"] == "evict":
        dq.dq_kv_evict(s["cache"], s["weights"], s["positions"], s["keep"], s["recent"], s["weights_out"], s["positions_out"],
                       s["lengths_out"], s["workspace"])
        return {"pages": s["pages"], "weights": s["weights_out"], "positions": s["positions_out"], "lengths": s["lengths_out"]}
    dq.dq_kv_attention(s["q"], s["cache"], s["scale"], s["out"], s["workspace"], starts=s["starts"], lse=s["sums"])
    return {"out": s["out"], "lse": s["sums"]}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------------------------------------------ 64 bits
def _held(s, b, h, n, second):
    """Keys (or values) of a sequence's first n slots in float64, slot by slot through the table."""
    dim, page = s["dim"], s["page"]
    slot = torch.arange(n, device="cuda")
    rows = s["pages"][s["table"][b][slot // page].long(), h]                       # a page's bytes for each slot
    base, token = slot % page // 16 * (16 * (dim + 8)) + second * 16 * (dim // 2 + 4), slot % 16
    code = (base + token * (dim // 2))[:, None] + torch.arange(dim, device="cuda") // 2
    byte = torch.gather(rows, 1, code).int()
    code = torch.where(torch.arange(dim, device="cuda") % 2 == 1, byte // 16, byte % 16).double()
    at = base + 16 * (dim // 2) + token * 4
    number = lambda i: ((torch.gather(rows, 1, (at + i)[:, None]).int()  # noqa: E731
                         + 256 * torch.gather(rows, 1, (at + i + 1)[:, None]).int()) << 16).view(torch.float32).double()
    return number(0) * code + number(2)


def _probabilities(s, b, h, group):
    """(probabilities, their sums' logarithm) [query][group][slot] of a sequence and a kv head."""
    first, last, n = (int(v) for v in (s["starts"][b], s["starts"][b + 1], s["lengths"][b]))
    q = s["q"][first:last, h * group:(h + 1) * group].double()
    logits = torch.einsum("igd,td->igt", q, _held(s, b, h, n, 0)) * s["scale"]
    later = torch.arange(n, device="cuda") > torch.arange(n - (last - first), n, device="cuda")[:, None]
    logits.masked_fill_(later[:, None], -math.inf)
    lse = torch.logsumexp(logits, -1)
    return logits.sub_(lse[..., None]).exp_(), lse


def _exact_rope(s, x, gamma):
    h = x.double()
    h = h / (h.square().sum(-1, keepdim=True) / h.shape[-1] + EPS).sqrt() * gamma.double()
    rot = s["rot"]
    i = torch.arange(0, rot // 2, device="cuda")
    a, b = (i, i + rot // 2) if s["pairs"] == "halves" else (2 * i, 2 * i + 1)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["inv_freq"].double())
    z = torch.complex(h[..., a], h[..., b]) * turn[:, None]
    h[..., a], h[..., b] = z.real, z.imag
    if s["hadamard"]:
        width = 1
        while width < h.shape[-1]:
            pair = h.unflatten(-1, (-1, 2, width))
            h = torch.stack((pair[..., 0, :] + pair[..., 1, :], pair[..., 0, :] - pair[..., 1, :]), -2).flatten(-3)
            width *= 2
        h = h / math.sqrt(h.shape[-1])
    return h


def _bf16_floor(v):
    """The largest bf16 value not above v (float64), by the spacing at its exponent."""
    step = torch.ldexp(torch.ones_like(v), torch.frexp(v).exponent.clamp(min=-125) - 8)
    return torch.floor(v / step) * step


def _exact_quantized(x):
    x = x.double()
    low = _bf16_floor(x.min(-1, keepdim=True).values)
    scale = -_bf16_floor(-(x.max(-1, keepdim=True).values - low) / 15)
    return torch.where(scale > 0, low + scale * torch.round((x - low) / scale), low)


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "rope":
        return {"q": _exact_rope(s, s["q"], s["q_gamma"]), "k": _exact_rope(s, s["k"], s["k_gamma"])}
    if s["op"] == "append":
        return {"pages": None, "keys": _exact_quantized(s["k"]), "values": _exact_quantized(s["v"])}
    if s["op"] == "evict":
        lengths, keep = s["lengths"].tolist(), s["keep"]
        for b, n in enumerate(lengths):
            for h in range(s["heads"]):
                w, pos = s["weights"][b, h, :n], s["positions"][b, h, :n]
                guarded = pos > pos.max() - s["recent"]
                order = torch.argsort(w.double(), descending=True, stable=True)
                order = torch.cat((order[guarded[order]].sort().values, order[~guarded[order]]))[:keep]
                inside = torch.zeros(n, dtype=torch.bool, device="cuda")
                inside[order] = True
                m = min(n, keep)
                src, dst = m + torch.nonzero(inside[m:])[:, 0], torch.nonzero(~inside[:m])[:, 0]
                where = torch.arange(m, device="cuda")
                where[dst] = src
                s["weights_out"][b, h, :m], s["positions_out"][b, h, :m] = w[where], pos[where]
        return {"pages": None, "weights": s["weights_out"].double(), "positions": None, "lengths": None}
    group = s["q_heads"] // s["heads"]
    starts, lengths = s["starts"].tolist(), s["lengths"].tolist()
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    sums = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    held = s["weights_out"].double() if s["op"] == "weights" else None
    for b, n in enumerate(lengths):
        rows = slice(starts[b], starts[b + 1])
        for h in range(s["heads"]):
            heads = slice(h * group, (h + 1) * group)
            p, lse = _probabilities(s, b, h, group)
            if held is not None:
                given = torch.exp(lse - s["lse"][rows, heads].double())[..., None]          # the sums that the call is given
                old = n - (starts[b + 1] - starts[b])
                held[b, h, :n] = (p * given).sum((0, 1))
                held[b, h, :old] += s["weights"][b, h, :old].double()
            else:
                out[rows, heads] = torch.einsum("igt,td->igd", p, _held(s, b, h, n, 1))
                sums[rows, heads] = lse
    return held if held is not None else {"out": out, "lse": sums}
