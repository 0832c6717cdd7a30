"""The paged-cache operators, as cases whose time can be measured and whose results can be compared.

A serving loop that compresses its caches at the end of a prefill still has to run that prefill, and the requests
that are not compressed, over a cache in pages.  One pass here is one call of

  append   queries and keys of a ragged batch rotated by their positions, keys and values stored into their pages
           (calidrop_paged_append)
  prefill  causal attention of a ragged batch of new tokens over the pages, with a sliding window and a few first tokens
           that stay visible (calidrop_paged_prefill)
  decode   the same for one new token a sequence (calidrop_paged_decode)
  prefix   one new token a sequence, where the sequences of a group share a long prefix whose pages are read once for all
           of them (calidrop_paged_prefix_decode)

`run` computes these in plain form, or with `own` set through the entry points of `paper_2507_19906_b200.binding`.

Inputs follow the statistics of `workload.py`: a base direction per query head that nearby queries share, unit-normal keys
and values, and a few first keys that point along the queries (attention sinks).  The pages of a sequence are scattered
over the pool.
"""
from __future__ import annotations

import math
import random
from types import SimpleNamespace

import torch

own = False

D = 128

_APPEND = dict(op="append", dtype="bf16", page=64, rot=128, interleaved=False, fused=False, positions=False)
_PREFILL = dict(op="prefill", dtype="bf16", page=64, window=0, sink=0)
_DECODE = dict(op="decode", dtype="bf16", page=64, window=0, sink=0)
_PREFIX = dict(op="prefix", dtype="bf16", page=64, groups=1)


def listed():
    return [
        # one decode step of a few requests: eight tokens into eight caches, a call that is all latency
        dict(_APPEND, name="append decode b8", Hq=32, Hkv=8, B=8, new=1, old=2048, mix=1),
        # one decode step of a full batch, half of the head rotated, in neighbouring pairs
        dict(_APPEND, name="append decode b256", Hq=32, Hkv=8, B=256, new=1, old=300, mix=2, page=16, rot=64, interleaved=True),
        # the prompts of a ragged batch, out of a fused projection's output, positions given by the caller
        dict(_APPEND, name="append ragged 16k", Hq=28, Hkv=4, B=7, new=2341, old=700, mix=3, dtype="fp16", fused=True, positions=True),
        # a short prompt, every key visible
        dict(_PREFILL, name="prefill 1k", Hq=32, Hkv=8, B=1, new=1024, old=0, mix=0),
        # an ordinary prompt, every key visible: the largest product
        dict(_PREFILL, name="prefill 8k", Hq=32, Hkv=8, B=1, new=8192, old=0, mix=0, page=128),
        # a long prompt through the sink-plus-recent cache of the paper's settings (32 sinks)
        dict(_PREFILL, name="prefill window 16k", Hq=16, Hkv=2, B=1, new=16384, old=0, mix=0, window=2016, sink=32),
        # chunks of several prompts on top of what their caches hold, from a single token to thousands, in fp16
        dict(_PREFILL, name="prefill ragged", Hq=28, Hkv=4, B=6, new=611, old=3001, mix=5, dtype="fp16", page=16, window=1500, sink=5),
        # one request, sinks and a short window: latency
        dict(_DECODE, name="decode window b1", Hq=32, Hkv=8, B=1, old=2111, mix=0, window=480, sink=32),
        # a batch of ragged caches, every key visible: the most bytes
        dict(_DECODE, name="decode b32", Hq=32, Hkv=8, B=32, old=8192, mix=6, page=16),
        # a batch of long caches, sinks and a window of which most of a cache is out of sight
        dict(_DECODE, name="decode window b48", Hq=40, Hkv=8, B=48, old=9000, mix=7, window=4064, sink=32, dtype="fp16"),
        # a few requests on one document
        dict(_PREFIX, name="prefix 8k b8", Hq=32, Hkv=8, B=8, prefix=8192, old=65, mix=8),
        # a full batch in three groups of unlike size, each on a long prefix of its own
        dict(_PREFIX, name="prefix 3x13k b96", Hq=32, Hkv=8, B=96, prefix=13001, old=301, mix=9, groups=3, page=32),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["append", "prefill", "decode", "prefix"])
    Hq, Hkv = rng.choice([(8, 8), (32, 8), (40, 8), (28, 4), (16, 2), (24, 8), (12, 4), (32, 32)])
    c = dict(op=op, Hq=Hq, Hkv=Hkv, dtype=rng.choice(["bf16", "bf16", "fp16"]), page=rng.choice([16, 32, 64, 128]),
             mix=rng.randint(1, 1 << 20))
    if op == "append":
        B = _log(rng, 1, 128)
        new = rng.choice([1, _log(rng, 1, 16384 // B)])
        while B * new * (Hq + 2 * Hkv) > 8 * 16384 * 8:
            new = new // 2 + 1
        return dict(c, B=B, new=new, old=_log(rng, 1, max(2, 65536 // B)), rot=rng.choice([128, 128, 64, 32, 96]), interleaved=rng.random() < 0.4,
                    fused=rng.random() < 0.4, positions=rng.random() < 0.3)
    c |= dict(window=rng.choice([0, _log(rng, 64, 4096)]), sink=rng.choice([0, 1, 4, 32, 130]))
    if op == "prefill":
        B, new, old = _log(rng, 1, 8), _log(rng, 16, 8192), rng.choice([0, _log(rng, 1, 8192)])
        while B * Hq * (2 * new) * (2 * new + 2 * old) > 32 * 8192 * 8192 * 2 // 3:
            new, old = new * 2 // 3 + 1, old * 2 // 3
        return dict(c, B=B, new=new, old=old)
    if op == "decode":
        B, old = _log(rng, 1, 64), _log(rng, 1, 32768)
        while B * Hkv * old > 32 * 8 * 8192 * 2 // 3:
            old = old * 2 // 3 + 1
        return dict(c, B=B, old=old)
    B, prefix, old = _log(rng, 1, 96), _log(rng, 128, 32768), _log(rng, 1, 300)
    groups = min(B, rng.choice([1, 1, 2, 4]))
    while groups * Hkv * prefix > 3 * 8 * 13001 or B * Hq * prefix > 96 * 32 * 13001:
        prefix = prefix * 2 // 3
    while B * Hkv * old > 96 * 8 * 301:
        old = old * 2 // 3 + 1
    c = {k: v for k, v in c.items() if k not in ("window", "sink")}
    return dict(c, B=B, prefix=prefix, old=old, groups=groups)


# ------------------------------------------------------------------------------------ sizes
def _spread(mean, n, mix, salt):
    """n whole numbers about `mean`, from a twelfth of it to twice as much (all of them `mean` for mix 0)."""
    if mix == 0:
        return [mean] * n
    rng = random.Random(mix * 7919 + salt)
    return [max(min(1, mean), int(mean * rng.choice([0.08, 0.3, 0.7, 1.0, 1.3, 1.62, 2.0]) * rng.uniform(0.9, 1.0))) for _ in range(n)]


def _sizes(c):
    """New tokens and cached rows of each sequence, the cached rows counting the new ones; group borders of a shared prefix."""
    B, mix = c["B"], c["mix"]
    new = _spread(c.get("new", 1), B, mix if c.get("new", 1) > 1 else 0, 1)
    if c["op"] == "prefill" and mix and B > 2:
        new[1] = 1                                        # a request that decodes, in the same batch
    old = _spread(c["old"], B, mix, 2)
    kv = [o + n for o, n in zip(old, new)] if c["op"] in ("append", "prefill") else [max(1, o) for o in old]
    s = SimpleNamespace(new=new, kv=kv, T=sum(new), borders=None, prefix=None)
    if c["op"] == "prefix":
        g = c["groups"]
        cuts = sorted(random.Random(mix).sample(range(1, B), g - 1)) if g > 1 else []
        s.borders = [0] + cuts + [B]
        s.prefix = [max(1, p) for p in _spread(c["prefix"], g, mix, 3)] if g > 1 else [c["prefix"]]
    return s


def _visible(n, window, sink, p):
    """Keys that the query at position p sees of the n that are cached."""
    keys = min(p + 1, n)
    return keys if not window or window >= keys else window + min(sink, keys - window)


def _pages(n, page):
    return (n + page - 1) // page


# ------------------------------------------------------------------------------------ inputs
def prepare(case, seed):
    c = case
    z = _sizes(c)
    B, Hq, Hkv, page, T = c["B"], c["Hq"], c["Hkv"], c["page"], z.T
    dt = {"bf16": torch.bfloat16, "fp16": torch.float16}[c["dtype"]]
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    s = SimpleNamespace(case=c, op=c["op"], T=T, page=page, window=c.get("window", 0), sink=c.get("sink", 0), Hq=Hq, Hkv=Hkv, G=Hq // Hkv)
    s.scale = 1.0 / math.sqrt(D)
    s.max_new, s.max_kv = max(z.new), max(z.kv)
    s.q_start = torch.tensor([sum(z.new[:i]) for i in range(B + 1)], dtype=torch.int32, device="cuda")
    s.kv_len = torch.tensor(z.kv, dtype=torch.int32, device="cuda")

    # the pool: each sequence's pages (and each prefix's) anywhere in it
    need = [_pages(n, page) for n in z.kv]
    pre_need = [_pages(n, page) for n in z.prefix] if z.prefix else []
    n_pages = sum(need) + sum(pre_need) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    max_pages = max(need)
    s.table = torch.zeros((B, max_pages), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        s.table[b, :n] = order[at:at + n]
        at += n
    s.K = torch.empty((n_pages, Hkv, page, D), dtype=dt, device="cuda")
    s.V = torch.empty_like(s.K)
    step = max(1, (1 << 26) // (Hkv * page * D))
    for i in range(0, n_pages, step):
        s.K[i:i + step] = normal(*s.K[i:i + step].shape)
        s.V[i:i + step] = normal(*s.V[i:i + step].shape)

    u = normal(Hq, D)                                     # the direction that a head's queries share
    if c["op"] == "append":
        s.rot, s.interleaved = c["rot"], c["interleaved"]
        s.max_pos = s.max_kv + 64
        angle = torch.arange(s.max_pos, dtype=torch.float64, device="cuda")[:, None] * \
            torch.pow(torch.tensor(10000.0, dtype=torch.float64, device="cuda"), -torch.arange(0, s.rot, 2, dtype=torch.float64, device="cuda") / s.rot)
        s.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().contiguous()
        rows = Hq + 2 * Hkv
        x = normal(T, rows, D)
        x[:, :Hq] = u + 0.3 * x[:, :Hq]
        x = x.to(dt)
        if c["fused"]:                                    # views into the projection's output
            s.q, s.k, s.v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        else:
            s.q, s.k, s.v = x[:, :Hq].contiguous(), x[:, Hq:Hq + Hkv].contiguous(), x[:, Hq + Hkv:].contiguous()
        s.positions = None
        if c["positions"]:
            s.positions = torch.randint(0, s.max_pos, (T,), generator=g, device="cuda", dtype=torch.int32)
        s.q_out = torch.empty((T, Hq, D), dtype=dt, device="cuda")
    else:
        s.q = (u + 0.3 * normal(T, Hq, D)).to(dt)
        s.out = torch.empty_like(s.q)
        s.lse = torch.empty((T, Hq), dtype=torch.float32, device="cuda")
        # attention sinks: the first keys of what a sequence sees point along the queries of their group
        first = s.table
        if c["op"] == "prefix":
            s.borders = torch.tensor(z.borders, dtype=torch.int32, device="cuda")
            s.prefix_len = torch.tensor(z.prefix, dtype=torch.int32, device="cuda")
            s.max_prefix, s.max_members = max(z.prefix), max(b - a for a, b in zip(z.borders, z.borders[1:]))
            s.prefix_table = torch.zeros((len(pre_need), max(pre_need)), dtype=torch.int32, device="cuda")
            for i, n in enumerate(pre_need):
                s.prefix_table[i, :n] = order[at:at + n]
                at += n
            first = s.prefix_table
        s.K[first[:, 0].long(), :, :4] = (0.5 * u.view(Hkv, -1, D).sum(1)).to(dt)[None, :, None, :]

    if own:
        from paper_2507_19906_b200 import binding as cd

        s.cd = cd
        s.p = cd.make_paged_params(B=B, Hq=Hq, Hkv=Hkv, dtype=dt, page_size=page, n_pages=n_pages, max_pages=max_pages, window=s.window, n_sink=s.sink,
                                   **(dict(rot_dim=s.rot, interleaved=s.interleaved, max_pos=s.max_pos, q_stride=s.q.stride(0),
                                           k_stride=s.k.stride(0), v_stride=s.v.stride(0)) if c["op"] == "append" else {}),
                                   **(dict(n_groups=c["groups"], max_prefix_pages=max(pre_need)) if c["op"] == "prefix" else {}))
        s.ws = torch.zeros((cd.calidrop_paged_workspace_bytes(s.p, T),), dtype=torch.uint8, device="cuda")
    return s


# ------------------------------------------------------------------------------------ one pass
def _own_append(s):
    s.cd.calidrop_paged_append(s.p, s.q, s.k, s.v, s.positions, s.cos_sin, s.K, s.V, s.table, s.q_start, s.kv_len, s.q_out, s.ws)
    return {"q": s.q_out, "K": s.K, "V": s.V}


def _own_prefill(s):
    s.cd.calidrop_paged_prefill(s.p, s.q, s.K, s.V, s.table, s.q_start, s.kv_len, s.out, s.lse, s.ws)
    return {"out": s.out, "lse": s.lse}


def _own_decode(s):
    s.cd.calidrop_paged_decode(s.p, s.q, s.K, s.V, s.table, s.kv_len, s.out, s.lse, s.ws)
    return {"out": s.out, "lse": s.lse}


def _own_prefix(s):
    s.cd.calidrop_paged_prefix_decode(s.p, s.q, s.K, s.V, s.borders, s.prefix_table, s.prefix_len, s.table, s.kv_len, s.out, s.lse, s.ws)
    return {"out": s.out, "lse": s.lse}


def _turn(x, cos, sin, interleaved):
    """x [T, H, rot] rotated by the angles whose cosines and sines are [T, rot / 2]."""
    cos, sin = cos[:, None], sin[:, None]
    if interleaved:
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, b * cos + a * sin], -1)


def _owner(start, n):
    """For n tokens in a row: the sequence that each belongs to, and its place in it."""
    t = torch.arange(n, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(start, t, right=True) - 1
    return b, t - start[b]


def _plain_append(s):
    b, i = _owner(s.q_start, s.T)
    at = s.kv_len[b] - (s.q_start[b + 1] - s.q_start[b]) + i
    cs = s.cos_sin[(at if s.positions is None else s.positions).long()]
    cos, sin = cs.chunk(2, 1)
    q, k = s.q.float(), s.k.float()
    s.q_out.copy_(torch.cat([_turn(q[..., :s.rot], cos, sin, s.interleaved), q[..., s.rot:]], -1))
    page, row = s.table[b, (at // s.page).long()].long(), (at % s.page).long()
    s.K[page, :, row] = torch.cat([_turn(k[..., :s.rot], cos, sin, s.interleaved), k[..., s.rot:]], -1).to(s.K.dtype)
    s.V[page, :, row] = s.v
    return {"q": s.q_out, "K": s.K, "V": s.V}


def _rows(pages, table, n):
    """The first n rows of each sequence, [B, Hkv, n, D] in 32 bits."""
    x = pages[table[:, :_pages(n, pages.shape[2])].long()].transpose(1, 2)
    return x.flatten(2, 3)[:, :, :n].float()


def _attend(q, K, V, mask, scale):
    """Parts of a softmax over masked keys: its maximum, its sum and the weighted values.  q [B, Hkv, G, M, D], K and V
    [B, Hkv, N, D], mask [B, M, N]."""
    B, H, G, M, _ = q.shape
    x = (q.reshape(B, H, G * M, D) @ K.transpose(-1, -2)).view(B, H, G, M, -1)
    x.mul_(scale).masked_fill_(~mask[:, None, None], -math.inf)
    m = x.amax(-1, keepdim=True).clamp_min(-1e30)
    x.sub_(m).exp_()
    l = x.sum(-1, keepdim=True)
    return m, l, (x.view(B, H, G * M, -1) @ V).view(B, H, G, M, D)


def _padded(q, start, most, s):
    """[T, Hq, D] -> [B, Hkv, G, most, D], and where each token went."""
    b, i = _owner(start, s.T)
    x = q.new_zeros((start.numel() - 1, most, s.Hq, D), dtype=torch.float32)
    x[b, i.long()] = q.float()
    return x.view(-1, most, s.Hkv, s.G, D).permute(0, 2, 3, 1, 4), b, i.long()


def _store(s, m, l, o):
    """Parts [T, Hkv, G, 1 or D] -> the outputs."""
    s.out.copy_((o / l.clamp_min(1e-38)).reshape(s.T, s.Hq, D))
    s.lse.copy_(torch.where(l > 0, m + l.log(), l.new_tensor(-math.inf)).reshape(s.T, s.Hq))
    return {"out": s.out, "lse": s.lse}


def _back(x, b, i):
    """[B, Hkv, G, M, .] -> [T, Hkv, G, .]"""
    return x.permute(0, 3, 1, 2, 4)[b, i]


def _plain_attention(s):
    q, b, i = _padded(s.q, s.q_start, s.max_new, s)
    t = torch.arange(s.max_kv, device="cuda", dtype=torch.int32)
    p = s.kv_len[:, None] - (s.q_start[1:] - s.q_start[:-1])[:, None] + torch.arange(s.max_new, device="cuda", dtype=torch.int32)
    mask = t <= p[:, :, None]
    if s.window:
        mask &= (t > p[:, :, None] - s.window) | (t < s.sink)
    parts = _attend(q, _rows(s.K, s.table, s.max_kv), _rows(s.V, s.table, s.max_kv), mask, s.scale)
    return _store(s, *(_back(x, b, i) for x in parts))


def _plain_prefix(s):
    q, b, i = _padded(s.q, s.borders, s.max_members, s)
    t = torch.arange(s.max_prefix, device="cuda", dtype=torch.int32)
    mask = (t < s.prefix_len[:, None, None]).expand(-1, s.max_members, -1)
    m1, l1, o1 = (_back(x, b, i) for x in _attend(q, _rows(s.K, s.prefix_table, s.max_prefix), _rows(s.V, s.prefix_table, s.max_prefix), mask, s.scale))
    t = torch.arange(s.max_kv, device="cuda", dtype=torch.int32)
    q = s.q.float().view(s.T, s.Hkv, s.G, 1, D)
    m2, l2, o2 = (x.squeeze(3) for x in _attend(q, _rows(s.K, s.table, s.max_kv), _rows(s.V, s.table, s.max_kv), t < s.kv_len[:, None, None], s.scale))
    m = torch.maximum(m1, m2)
    f1, f2 = (m1 - m).exp(), (m2 - m).exp()
    return _store(s, m, l1 * f1 + l2 * f2, o1 * f1 + o2 * f2)


def run(state):
    if own:
        return {"append": _own_append, "prefill": _own_prefill, "decode": _own_decode, "prefix": _own_prefix}[state.op](state)
    return {"append": _plain_append, "prefill": _plain_attention, "decode": _plain_attention, "prefix": _plain_prefix}[state.op](state)


# ------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    c, z = case, _sizes(case)
    Hq, Hkv, T = c["Hq"], c["Hkv"], z.T
    row = 2 * D                                           # bytes of one head's row
    if c["op"] == "append":
        # q, k, v in; q, k, v out; the angles of each token; tables
        return {"bytes": 2 * T * (Hq + 2 * Hkv) * row + 4 * T * c["rot"], "flops": 3 * T * (Hq + Hkv) * c["rot"]}
    window, sink = c.get("window", 0), c.get("sink", 0)
    pairs = rows = 0
    if c["op"] == "prefix":
        for a, b, n in zip(z.borders, z.borders[1:], z.prefix):
            pairs += (b - a) * n
            rows += n
        pairs += sum(z.kv)
        rows += sum(z.kv)
    else:
        for n, kv in zip(z.new, z.kv):
            pairs += sum(_visible(kv, window, sink, p) for p in range(kv - n, kv))
            # the keys that any of its queries sees
            lo = max(0, kv - n - window + 1) if window else 0
            rows += min(kv, kv - lo + min(sink, lo))
    return {"bytes": 2 * rows * Hkv * row + 2 * T * Hq * row + 4 * T * Hq, "flops": 4 * pairs * Hq * D}


# ------------------------------------------------------------------------------------ the definition, in 64 bits
def exact(case, seed):
    s, z = prepare(case, seed), _sizes(case)
    if s.op == "append":
        K, V, Q = s.K.double(), s.V.double(), s.q.double().clone()
        tok = 0
        for b, (n, kv) in enumerate(zip(z.new, z.kv)):
            at = torch.arange(kv - n, kv, device="cuda")
            sl = slice(tok, tok + n)
            pos = at if s.positions is None else s.positions[sl].long()
            w = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.zeros((), dtype=torch.float64, device="cuda"))
            w = w * torch.complex(s.cos_sin[pos, :s.rot // 2].double(), s.cos_sin[pos, s.rot // 2:].double())[:, None]
            k = s.k[sl].double().clone()
            for x in (Q[sl], k):                          # each pair is a complex number, turned by the token's
                if s.interleaved:
                    y = torch.view_as_complex(x[..., :s.rot].unflatten(-1, (-1, 2)).contiguous()) * w
                    x[..., 0:s.rot:2], x[..., 1:s.rot:2] = y.real, y.imag
                else:
                    y = torch.complex(x[..., :s.rot // 2], x[..., s.rot // 2:s.rot]) * w
                    x[..., :s.rot // 2], x[..., s.rot // 2:s.rot] = y.real, y.imag
            page = s.table[b].long()[at // s.page]
            K[page, :, at % s.page] = k
            V[page, :, at % s.page] = s.v[sl].double()
            tok += n
        return {"q": Q, "K": K, "V": V}

    out = torch.empty((s.T, s.Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.empty((s.T, s.Hq), dtype=torch.float64, device="cuda")

    def cached(x, table, n, h):
        return x[table[:_pages(n, s.page)].long(), h].reshape(-1, D)[:n].double()

    tok = 0
    for b, (n, kv) in enumerate(zip(z.new, z.kv)):
        for h in range(s.Hkv):
            K, V = cached(s.K, s.table[b], kv, h), cached(s.V, s.table[b], kv, h)
            pre = 0
            if s.op == "prefix":
                group = sum(b >= e for e in z.borders[1:])
                pre = z.prefix[group]
                K = torch.cat([cached(s.K, s.prefix_table[group], pre, h), K])
                V = torch.cat([cached(s.V, s.prefix_table[group], pre, h), V])
            for i0 in range(0, n, 2048):
                i1 = min(n, i0 + 2048)
                p = torch.arange(pre + kv - n + i0, pre + kv - n + i1, device="cuda")[:, None]
                t = torch.arange(K.shape[0], device="cuda")
                seen = (t <= p) & (((p - t) < s.window) | (t < s.sink) if s.window else t >= 0)
                for hq in range(h * s.G, (h + 1) * s.G):
                    x = torch.where(seen, s.q[tok + i0:tok + i1, hq].double() @ K.T / math.sqrt(D), -math.inf)
                    lse[tok + i0:tok + i1, hq] = torch.logsumexp(x, 1)
                    out[tok + i0:tok + i1, hq] = torch.softmax(x, 1) @ V
        tok += n
    return {"out": out, "lse": lse}
