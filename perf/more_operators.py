"""Performance cases of the attention behind the norm and rotation of queries and
keys, and of the key and value cache that serving reads.

Four kinds of call, with ``own`` through the package's public Python entry
points, without it in elementary torch operations:

* ``attn``     causal attention of packed sequences with a sliding window and a
  few first tokens that stay visible (sinks), or without a window; queries may
  be the last ones of their keys (a chunk of a prompt);
* ``attnbwd``  its gradients: queries, keys, values;
* ``append``   new tokens' keys and values into a paged cache;
* ``cached``   attention of new tokens over the cache: one a sequence, or a tree
  of drafted tokens, each with a bit mask of the drafted ones it sees; the cache
  in bf16 or in E4M3 codes with a power-of-two scale for 32 elements.

Heads are N(0, 1) as a norm leaves them, queries 1.5 times that, output
gradients 0.01 N(0, 1).
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"


def listed():
    return [
        # a chunk of 129 prompt tokens behind 383 that the layer has kept: latency
        dict(name="attn_chunk", op="attn", T=129, seqs=1, kept=383, Hq=8, Hk=2, D=64, window=256, sinks=4, train=False),
        # a small model's batch of packed sequences, odd sizes everywhere
        dict(name="attn_ragged", op="attn", T=5003, seqs=9, kept=0, Hq=12, Hk=4, D=80, window=1000, sinks=5, train=True),
        # an 8B model's layer over one 8k sequence, no window: the largest forward
        dict(name="attn_train8k", op="attn", T=8192, seqs=1, kept=0, Hq=32, Hk=8, D=128, window=0, sinks=0, train=True),
        # one 1024-token step of a 125M-parameter model: launches and latency
        dict(name="attnbwd_125m", op="attnbwd", T=1024, seqs=1, kept=0, Hq=12, Hk=12, D=64, window=0, sinks=0),
        # packed sequences with a window and sinks, odd sizes everywhere
        dict(name="attnbwd_ragged", op="attnbwd", T=3001, seqs=7, kept=0, Hq=8, Hk=2, D=96, window=500, sinks=3),
        # an 8B model's layer over one 8k sequence with a window: the largest call
        dict(name="attnbwd_8k", op="attnbwd", T=8192, seqs=1, kept=0, Hq=32, Hk=8, D=128, window=4096, sinks=4),
        # one decoding step of 61 sequences: latency
        dict(name="append_decode61", op="append", seqs=61, new=1, longest=2048, page=16, Hk=8, D=128, rows=False),
        # prompts of 16384 tokens in all into the cache: bandwidth
        dict(name="append_prefill16k", op="append", seqs=4, new=4096, longest=512, page=64, Hk=8, D=128, rows=False),
        # one token behind 128k: few heads, the key axis alone to share out
        dict(name="cached_long1", op="cached", elem="bf16", seqs=1, new=1, tree=False, longest=131072, page=64, Hq=32,
             Hk=8, D=128, window=0, sinks=0),
        # one decoding step of 61 sequences of up to 16k tokens, an 8-bit cache
        dict(name="cached_decode61_mx", op="cached", elem="e4m3", seqs=61, new=1, tree=False, longest=16384, page=32, Hq=32,
             Hk=8, D=128, window=0, sinks=0),
        # drafted trees of up to 63 tokens behind 16 sequences
        dict(name="cached_tree16", op="cached", elem="bf16", seqs=16, new=63, tree=True, longest=8192, page=16, Hq=32, Hk=8,
             D=128, window=0, sinks=0),
        # a small model's step that reads sinks and a window of long sequences: the smallest
        dict(name="cached_window16", op="cached", elem="bf16", seqs=16, new=1, tree=False, longest=20000, page=16, Hq=12,
             Hk=4, D=64, window=1024, sinks=4),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case: a kind by its weight, sizes log-uniform over the range."""
    op = rng.choice(["attn", "attn", "attnbwd", "attnbwd", "append", "cached", "cached", "cached"])
    Hk = rng.choice([1, 2, 4, 8, 8])
    G = rng.choice([1, 2, 3, 4, 4, 8])
    G = min(G, 32 // Hk)
    if op in ("attn", "attnbwd"):
        D = rng.choice([64, 72, 80, 96, 128, 128])
        T = rng.choice([_log(rng, 64, 1024), _log(rng, 1024, 8192)])
        kept = _log(rng, 16, 1024) if op == "attn" and T < 2048 and rng.random() < 0.4 else 0
        window = rng.choice([0, _log(rng, 32, 4096), _log(rng, 32, 4096)])
        case = dict(op=op, T=T, seqs=rng.choice([1, 1, _log(rng, 2, 16)]), kept=kept, Hq=Hk * G, Hk=Hk, D=D, window=window,
                    sinks=rng.choice([0, 1, 4, 16]) if window else 0)
        if op == "attn":
            case["train"] = rng.choice([False, True])
        return case
    if op == "append":
        seqs = _log(rng, 1, 128)
        return dict(op=op, seqs=seqs, new=_log(rng, 1, 16384 // seqs), longest=_log(rng, 16, 4096), page=rng.choice([16, 32, 64, 256]),
                    Hk=Hk, D=rng.choice([64, 80, 96, 128, 128]), rows=rng.choice([False, True]))
    tree = rng.random() < 0.4
    seqs, new = _log(rng, 1, 64), rng.choice([1, 1, _log(rng, 2, 63)])
    if tree:
        seqs, new = _log(rng, 1, 16), _log(rng, 3, 63)
    window = rng.choice([0, 0, _log(rng, 64, 4096)])
    return dict(op=op, elem=rng.choice(["bf16", "e4m3"]), seqs=seqs, new=new, tree=tree,
                longest=_log(rng, 16, min(131072, 16 * 8192 * 63 * 32 // (seqs * new * Hk * G), 61 * 16384 // seqs)),
                page=rng.choice([16, 32, 64, 256]), Hq=Hk * G, Hk=Hk, D=rng.choice([64, 96, 128, 128]), window=window,
                sinks=rng.choice([0, 4]) if window else 0)


# ------------------------------------------------------------------- sizes --

def _lengths(total, n):
    """n uneven lengths that add up to total."""
    weight = [1 + i * 5 % 7 for i in range(n)]
    ends = [total * sum(weight[:i]) // sum(weight) for i in range(n + 1)]
    return [b - a for a, b in zip(ends, ends[1:])]


def _contexts(case):
    """Tokens in the cache and new ones of every sequence."""
    n, far = case["seqs"], case["longest"]
    cached = [far - far * (b * 5 % 8) // 10 for b in range(n)]
    ragged = case["new"] > 1 and case["op"] == "cached"
    return cached, [max(1, case["new"] - b * 3 % 5) if ragged else case["new"] for b in range(n)]


def _starts(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(torch.int32).to(DEV)


# ------------------------------------------------------------------ inputs --

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device=DEV, dtype=torch.bfloat16)


def _cache(c, g, elem):
    """A cache of pages [pages, heads, slots, D] and every sequence's pages."""
    cached, new = _contexts(c)
    page, need = c["page"], [-(-(a + b) // c["page"]) for a, b in zip(cached, new)]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32).cpu()
    table = torch.full((c["seqs"], max(need) + 1), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    c["table"], c["length"] = table.to(DEV), torch.tensor(cached, dtype=torch.int32, device=DEV)
    c["start"] = _starts(new)
    c["kc"], c["vc"] = [_normal(g, pages, c["Hk"], page, c["D"]) for _ in range(2)]
    c["ks"] = c["vs"] = None
    if elem == "e4m3":
        c["kc"], c["ks"] = _encode(c["kc"])
        c["vc"], c["vs"] = _encode(c["vc"])


def _encode(t):
    """E4M3 codes and E8M0 scale bytes of blocks of 32 along the last axis: the
    smallest power of two under which nothing passes 448."""
    v = t.float().unflatten(-1, (-1, 32))
    e = (((v.abs().amax(-1).view(torch.int32) + 0x1FFFFF) >> 23) - 8).clamp(min=1)
    codes = (v * ((254 - e) << 23).view(torch.float32)[..., None]).flatten(-2).to(torch.float8_e4m3fn)
    return codes.view(torch.uint8), e.to(torch.uint8)


def _tree(case, seed):
    """Bit i of a token's mask: it sees its sequence's drafted token i."""
    g = torch.Generator().manual_seed(seed)
    n = case["new"]
    parent = (torch.rand(case["seqs"], n, generator=g) * (torch.arange(n) + 1)).long() - 1
    bits = torch.zeros(case["seqs"], n + 1, dtype=torch.int64)  # the last: no parent
    for i in range(n):
        bits[:, i] = (1 << i) | bits.gather(1, parent[:, i:i + 1] % (n + 1))[:, 0]
    return torch.cat([bits[b, :m] for b, m in enumerate(_contexts(case)[1])]).to(DEV)


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    c, op, Hk, D = dict(case), case["op"], case["Hk"], case["D"]
    if op in ("append", "cached"):
        _cache(c, g, c.get("elem", "bf16"))
        T = sum(_contexts(c)[1])
        if op == "append":
            # the fused projection's keys and values; after drafts, rows of those kept
            kv = _normal(g, 2 * T if c["rows"] else T, 2 * Hk * D)
            c["k"], c["v"] = kv[:, :Hk * D].unflatten(1, (Hk, D)), kv[:, Hk * D:].unflatten(1, (Hk, D))
            c["rows"] = torch.randperm(2 * T, generator=g, device=DEV)[:T].to(torch.int32) if c["rows"] else None
        else:
            c["q"] = 1.5 * _normal(g, T, c["Hq"], D)
            c["bits"] = _tree(case, seed) if c["tree"] else None
        return c
    T, Hq = c["T"], c["Hq"]
    queries = _lengths(T, c["seqs"])
    keys = [n + c["kept"] for n in queries]
    c["q_start"], c["k_start"] = _starts(queries), _starts(keys)
    # views of a projection's output where queries and keys are the same tokens
    S = sum(keys)
    if c["kept"]:
        c["q"], c["k"], c["v"] = 1.5 * _normal(g, T, Hq, D), _normal(g, S, Hk, D), _normal(g, S, Hk, D)
    else:
        qkv = _normal(g, T, (Hq + 2 * Hk), D)
        qkv[:, :Hq] *= 1.5
        c["q"], c["k"], c["v"] = qkv.split([Hq, Hk, Hk], 1)
    if op == "attnbwd":
        c["go"] = 0.01 * _normal(g, T, Hq, D)
        # what the forward of this step kept
        c["o"], c["lse"] = _attention(c)
        # where the gradient of the projection's output is collected
        c["gq"], c["gk"], c["gv"] = torch.zeros_like(qkv).split([Hq, Hk, Hk], 1)
    return c


# -------------------------------------------------- the operators, plainly --

def _visible(s):
    """[queries, keys]: which keys a query sees."""
    T, S = s["q"].shape[0], s["k"].shape[0]
    qs, ks = s["q_start"].long(), s["k_start"].long()
    i, j = torch.arange(T, device=DEV), torch.arange(S, device=DEV)
    a, b = torch.searchsorted(qs, i, right=True) - 1, torch.searchsorted(ks, j, right=True) - 1
    # positions in the sequence: the queries are its last ones
    p = (i - qs[a + 1] + ks[a + 1] - ks[a])[:, None]
    j = (j - ks[b])[None]
    seen = (a[:, None] == b[None]) & (j <= p)
    if s["window"]:
        seen &= (p - j < s["window"]) | (j < s["sinks"])
    return seen


def _by_group(t, Hk):
    """[T, heads, D] as float32 [Hk, heads of the group x T, D]."""
    T, H, D = t.shape
    return t.float().view(T, Hk, H // Hk, D).permute(1, 2, 0, 3).reshape(Hk, -1, D)


def _ungroup(t, T):
    Hk, n, D = t.shape
    return t.view(Hk, n // T, T, D).permute(2, 0, 1, 3).reshape(T, -1, D)


def _scores(s):
    """Masked scores [Hk, heads of the group, queries, keys] of the grouped heads."""
    T, Hk = s["q"].shape[0], s["Hk"]
    x = _by_group(s["q"], Hk) @ _by_group(s["k"], Hk).transpose(1, 2)
    x = x.mul_(s["D"] ** -0.5).view(Hk, -1, T, x.shape[-1])
    return x.masked_fill_(~_visible(s), -math.inf)


def _attention(s):
    T, Hk = s["q"].shape[0], s["Hk"]
    x = _scores(s)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m.masked_fill(m == -math.inf, 0)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.flatten(1, 2) @ _by_group(s["v"], Hk)) / total.flatten(1, 2).clamp(min=1e-30)
    return _ungroup(o, T).bfloat16(), (m + total.log()).view(s["Hq"], T)


def _attention_gradient(s):
    T, Hk, scale = s["q"].shape[0], s["Hk"], s["D"] ** -0.5
    p = _scores(s).sub_(s["lse"].view(Hk, -1, T, 1)).exp_().flatten(1, 2)
    q, k, v, go = (_by_group(s[n], Hk) for n in ("q", "k", "v", "go"))
    gv = p.transpose(1, 2) @ go
    delta = (go * _by_group(s["o"], Hk)).sum(-1, keepdim=True)
    ds = (go @ v.transpose(1, 2)).sub_(delta).mul_(p).mul_(scale)
    for to, t in ((s["gq"], _ungroup(ds @ k, T)), (s["gk"], (ds.transpose(1, 2) @ q).transpose(0, 1)), (s["gv"], gv.transpose(0, 1))):
        to.copy_(t)
    return s["gq"], s["gk"], s["gv"]


def _append(s):
    start, T = s["start"].long(), s["k"].shape[0] if s["rows"] is None else s["rows"].shape[0]
    t = torch.arange(T, device=DEV)
    b = torch.searchsorted(start, t, right=True) - 1
    at = s["length"].long()[b] + t - start[b]
    page, slot = s["table"].long()[b, at // s["page"]], at % s["page"]
    rows = slice(None) if s["rows"] is None else s["rows"].long()
    s["kc"][page, :, slot] = s["k"][rows]
    s["vc"][page, :, slot] = s["v"][rows]
    return s["kc"], s["vc"]


def _read(s, codes, scales, page, slot):
    """float32 [sequences, heads, keys, D] of the cache's slots."""
    x = codes[page, :, slot]
    if scales is None:
        return x.float().transpose(1, 2).contiguous()
    x = x.view(torch.float8_e4m3fn).float().unflatten(-1, (-1, 32))
    x.mul_((scales[page, :, slot].int() << 23).view(torch.float32)[..., None])
    return x.flatten(-2).transpose(1, 2).contiguous()


def _cached(s):
    B, T, Hk, D = s["seqs"], s["q"].shape[0], s["Hk"], s["D"]
    cached, new = _contexts(s)
    keys, most = max(a + b for a, b in zip(cached, new)), max(new)
    start, length = s["start"].long(), s["length"].long()
    j = torch.arange(keys, device=DEV)
    page = s["table"].long()[:, j // s["page"]].clamp(min=0)
    k, v = (_read(s, s[a], s[b], page, j % s["page"]) for a, b in (("kc", "ks"), ("vc", "vs")))
    # queries by sequence, the shorter ones filled up with their last
    i = torch.arange(most, device=DEV)
    n = start[1:] - start[:-1]
    t = start[:-1, None] + torch.minimum(i[None], n[:, None] - 1)
    q = s["q"][t].float().view(B, most, Hk, -1, D).permute(0, 2, 3, 1, 4).reshape(B, Hk, -1, D)
    x = (q @ k.transpose(2, 3)).mul_(D ** -0.5).view(B, Hk, -1, most, keys)
    # a token's mask of the drafted ones, and from it its place
    bits = s["bits"][t] if s["bits"] is not None else ((2 << i) - 1).expand(B, most)
    own_bits = bits[..., None] >> torch.arange(most, device=DEV) & 1
    place = length[:, None] + own_bits.sum(-1) - 1
    drafted = (j[None] - length[:, None]).clamp(0, most - 1)
    old = j[None] < length[:, None]
    at = torch.where(old, j[None], place.gather(1, drafted))
    seen = old[:, None] | (own_bits.gather(2, drafted[:, None].expand(B, most, keys)) == 1)
    seen &= (j[None] < (length + n)[:, None])[:, None]
    if s["window"]:
        seen &= (place[..., None] - at[:, None] < s["window"]) | (at < s["sinks"])[:, None]
    x.masked_fill_(~seen[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True)
    p = x.sub_(m.masked_fill(m == -math.inf, 0)).exp_()
    o = p.flatten(2, 3) @ v / p.sum(-1).flatten(2)[..., None].clamp(min=1e-30)
    o = o.view(B, Hk, -1, most, D).permute(0, 3, 1, 2, 4).reshape(B, most, -1, D).bfloat16()
    of = torch.searchsorted(start, torch.arange(T, device=DEV), right=True) - 1
    return o[of, torch.arange(T, device=DEV) - start[of]]


def _plain(s):
    op = s["op"]
    if op == "attn":
        o, lse = _attention(s)
        return (o, lse) if s["train"] else o
    return {"attnbwd": _attention_gradient, "append": _append, "cached": _cached}[op](s)


def run(s):
    if not own:
        return _plain(s)
    from paper_2603_13180_amd import mxnorm
    op = s["op"]
    if op == "append":
        return mxnorm.kv_cache_append(s["k"], s["v"], s["kc"], s["vc"], s["table"], s["length"], start=s["start"], rows=s["rows"])
    if op == "cached":
        return mxnorm.kv_cache_attn_fwd(s["q"], s["kc"], s["vc"], s["table"], s["length"], k_scales=s["ks"], v_scales=s["vs"],
                                        start=s["start"], max_new=s["new"], ancestors=s["bits"], window=s["window"],
                                        sinks=s["sinks"])
    kw = dict(window=s["window"], sinks=s["sinks"], q_start=s["q_start"], k_start=s["k_start"] if s["kept"] else None)
    if op == "attn":
        o, lse = mxnorm.window_attn_fwd(s["q"], s["k"], s["v"], want_lse=s["train"], **kw)
        return (o, lse) if s["train"] else o
    return mxnorm.window_attn_bwd(s["go"], s["q"], s["k"], s["v"], s["o"], s["lse"], grad_q=s["gq"], grad_k=s["gk"],
                                  grad_v=s["gv"], **kw)


# -------------------------------------------------------------------- work --

def _seen_by(place, window, sinks):
    """How many keys a token at this place of its sequence sees."""
    n = place + 1
    return n if not window else np.minimum(n, window + np.minimum(sinks, np.maximum(n - window, 0)))


def work(case):
    op, Hk, D = case["op"], case["Hk"], case["D"]
    if op in ("append", "cached"):
        cached, new = _contexts(case)
        T = sum(new)
        if op == "append":
            return {"bytes": 8 * T * Hk * D + 4 * len(new), "flops": T * Hk * D}
        element = 2 if case["elem"] == "bf16" else 33 / 32
        keys = sum(int(_seen_by(np.int64(a + b - 1), case["window"], case["sinks"])) for a, b in zip(cached, new))
        pairs = sum(b * int(_seen_by(np.int64(a + b // 2), case["window"], case["sinks"])) for a, b in zip(cached, new))
        return {"bytes": int(2 * keys * Hk * D * element) + 4 * T * case["Hq"] * D, "flops": 4 * pairs * case["Hq"] * D}
    T, Hq = case["T"], case["Hq"]
    S, pairs = T + case["seqs"] * case["kept"], 0
    for n in _lengths(T, case["seqs"]):
        pairs += int(_seen_by(np.arange(n, dtype=np.int64) + case["kept"], case["window"], case["sinks"]).sum())
    if op == "attn":
        return {"bytes": 4 * T * Hq * D + 4 * S * Hk * D + (4 * T * Hq if case["train"] else 0), "flops": 4 * pairs * Hq * D}
    return {"bytes": 8 * T * Hq * D + 8 * S * Hk * D + 4 * T * Hq, "flops": 10 * pairs * Hq * D}


# ------------------------------------------------------- the same in 64 bits --

def _softmax_values(x, seen, v):
    """(softmax over the seen keys times v, log of the sum of exponentials)."""
    x = x.masked_fill(~seen, -1e300)
    p = torch.softmax(x, -1) * seen
    return p @ v, torch.logsumexp(x, -1)


def _exact_attention(s):
    """Output, lse and, with an output gradient, the gradients, by sequence and head."""
    q, k, v = (s[n].double() for n in ("q", "k", "v"))
    (T, Hq, D), Hk = q.shape, k.shape[1]
    back = s["op"] == "attnbwd"
    o, lse = torch.zeros_like(q), torch.empty(Hq, T, dtype=torch.float64, device=DEV)
    grads = [torch.zeros_like(t) for t in (q, k, v)]
    qs, ks = s["q_start"].tolist(), s["k_start"].tolist()
    for a, b, c, d in zip(qs, qs[1:], ks, ks[1:]):
        p, j = torch.arange(d - c - (b - a), d - c, device=DEV)[:, None], torch.arange(d - c, device=DEV)
        seen = (j <= p) if not s["window"] else (j <= p) & ((j > p - s["window"]) | (j < s["sinks"]))
        for h in range(Hq):
            leaf = [t.clone().requires_grad_(back) for t in (q[a:b, h], k[c:d, h * Hk // Hq], v[c:d, h * Hk // Hq])]
            out, total = _softmax_values(leaf[0] @ leaf[1].t() / math.sqrt(D), seen, leaf[2])
            if back:
                for t, x in zip(grads, torch.autograd.grad(out, leaf, s["go"][a:b, h].double())):
                    t[slice(a, b) if t is grads[0] else slice(c, d), h if t is grads[0] else h * Hk // Hq] += x
            else:
                o[a:b, h], lse[h, a:b] = out, total
    return grads if back else (o, lse)


def _exact_slots(codes, scales, pages):
    """float64 [heads, keys, D] of whole pages, code by code."""
    x = codes[pages].transpose(0, 1).flatten(1, 2)
    if scales is None:
        return x.double()
    x = x.int()
    e, m = x >> 3 & 15, (x & 7).double() / 8
    y = torch.where(e == 0, m * 2.0 ** -6, torch.ldexp(1 + m, e - 7)) * torch.where(x > 127, -1.0, 1.0)
    return torch.ldexp(y, (scales[pages].transpose(0, 1).flatten(1, 2).int() - 127).repeat_interleave(32, -1))


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op in ("attn", "attnbwd"):
        got = _exact_attention(s)
        return got if op == "attnbwd" or case["train"] else got[0]
    table, start, length = s["table"].tolist(), s["start"].tolist(), s["length"].tolist()
    if op == "append":
        for b, n in enumerate(length):
            t = torch.arange(start[b], start[b + 1], device=DEV)
            place = n + t - start[b]
            page, row = s["table"][b].long()[place // case["page"]], t if s["rows"] is None else s["rows"].long()[t]
            s["kc"].transpose(1, 2)[page, place % case["page"]] = s["k"][row]
            s["vc"].transpose(1, 2)[page, place % case["page"]] = s["v"][row]
        return s["kc"].double(), s["vc"].double()
    q, group = s["q"].double(), case["Hq"] // case["Hk"]
    o = torch.empty_like(q)
    for b, n in enumerate(length):
        mine = slice(start[b], start[b + 1])
        new = start[b + 1] - start[b]
        pages = torch.tensor([p for p in table[b] if p >= 0], device=DEV)
        k, v = (_exact_slots(s[x], s[y], pages)[:, :n + new] for x, y in (("kc", "ks"), ("vc", "vs")))
        drafted = torch.ones(new, new, dtype=torch.bool, device=DEV).tril()
        if s["bits"] is not None:
            drafted = s["bits"][mine, None].bitwise_and(1 << torch.arange(new, device=DEV)) != 0
        place = n - 1 + drafted.sum(1)
        at = torch.cat((torch.arange(n, device=DEV), place))
        seen = torch.cat((torch.ones(new, n, dtype=torch.bool, device=DEV), drafted), 1)
        if case["window"]:
            seen = seen & ((at > place[:, None] - case["window"]) | (at < case["sinks"]))
        x = q[mine].transpose(0, 1).unflatten(0, (-1, group)) @ k.transpose(1, 2)[:, None].contiguous() / math.sqrt(case["D"])
        o[mine] = _softmax_values(x, seen, v[:, None].contiguous())[0].flatten(0, 1).transpose(0, 1)
    return o
