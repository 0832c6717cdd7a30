"""Caches in pages for the tests, and the definitions of the operators over them in 64 bits (plain loops, torch on the CPU or GPU)."""
from __future__ import annotations

import math
from types import SimpleNamespace

import torch

from paper_2507_19906_b200 import binding as cd

D = 128
HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step of a rounding, relative to the value
# ... and at least this: values below the smallest normal one (2^-14 in fp16) lie a fixed step apart, 2^-24 = 2^-14 * 2^-10 (in
# bf16 2^-126 * 2^-7).  6.86e-6 in fp16, for one, is 115.2 steps, and rounds by 0.2 of a step where 2^-11 of the value is 0.056.
SMALL = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def n_pages_of(n, page):
    return (n + page - 1) // page


class Pool:
    """A pool of pages in scattered order.  Rows that no sequence has written hold NaN."""

    def __init__(self, lens, *, Hkv, page, dtype=torch.bfloat16, seed=0, interleaved_pool=False, spare=3, max_pages=None, scale=1.0):
        self.lens, self.Hkv, self.page, self.dtype = list(lens), Hkv, page, dtype
        g = torch.Generator().manual_seed(seed)
        need = [n_pages_of(n, page) for n in lens]
        self.n_pages = sum(need) + spare
        order = torch.randperm(self.n_pages, generator=g).to(torch.int32)
        self.max_pages = max_pages or max(1, max(need, default=1))
        table = torch.full((max(1, len(lens)), self.max_pages), -1, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        shape = (self.n_pages, Hkv, page, D)
        if interleaved_pool:
            both = torch.full((self.n_pages, 2, Hkv, page, D), math.nan, dtype=dtype, device="cuda")
            self.K, self.V = both[:, 0], both[:, 1]
            self.page_stride = both.stride(0)
        else:
            self.K = torch.full(shape, math.nan, dtype=dtype, device="cuda")
            self.V = torch.full(shape, math.nan, dtype=dtype, device="cuda")
            self.page_stride = 0
        self.k_rows = [(scale * torch.randn((Hkv, n, D), generator=g)).to(dtype).cuda() for n in lens]
        self.v_rows = [torch.randn((Hkv, n, D), generator=g).to(dtype).cuda() for n in lens]
        self.table = table.cuda()
        for b, n in enumerate(lens):
            self.write(b, 0, self.k_rows[b], self.v_rows[b])

    def write(self, b, t0, k, v):
        n = k.shape[1]
        if n == 0:
            return
        t = torch.arange(t0, t0 + n, device="cuda")
        pg = self.table[b, (t // self.page).long()].long()
        self.K[pg, :, t % self.page] = k.transpose(0, 1)
        self.V[pg, :, t % self.page] = v.transpose(0, 1)

    def read(self, x, b, n):
        """Rows [0, n) of sequence b: [Hkv, n, D]."""
        t = torch.arange(n, device="cuda")
        return x[self.table[b, (t // self.page).long()].long(), :, t % self.page].transpose(0, 1)

    def hide(self, b, window, n_sink, lo_pos):
        """Forget the pages of which no query at or behind position lo_pos sees a row: their entries become -1."""
        for i in range(n_pages_of(self.lens[b], self.page)):
            first, last = i * self.page, (i + 1) * self.page - 1
            if first >= n_sink and last <= lo_pos - window:
                self.table[b, i] = -1


def visible(p, kv, window, n_sink):
    """[len(p), kv] of truth values."""
    t = torch.arange(kv, device=p.device)
    s = t <= p[:, None]
    if window:
        s &= (t > p[:, None] - window) | (t < n_sink)
    return s


def attention64(q, k, v, seen, scale):
    """q [M, D], k, v [N, D], seen [M, N] -> out, lse, and what errors are measured by: sum p |v| and the largest sum of |q k|."""
    q, k, v = q.double(), k.double(), v.double()
    if k.shape[0] == 0:
        z = torch.zeros((q.shape[0], D), dtype=torch.float64, device=q.device)
        return z, torch.full((q.shape[0],), -math.inf, dtype=torch.float64, device=q.device), z, z[:, 0]
    x = torch.where(seen, q @ k.T * scale, -math.inf)
    lse = torch.logsumexp(x, 1)
    p = torch.where(seen, torch.exp(x - torch.where(torch.isfinite(lse), lse, torch.zeros_like(lse))[:, None]), 0.0)
    any_key = seen.any(1)
    sizes = torch.where(seen, q.abs() @ k.abs().T * scale, 0.0).amax(1)
    out = torch.where(any_key[:, None], p @ v, 0.0)
    return out, torch.where(any_key, lse, -math.inf), p @ v.abs(), sizes


def check_rows(out, lse, ref, dtype, n_keys, what=""):
    """Outputs against the definition's.  An output is off by its own rounding (half a step of its value), by the rounding of the
    probabilities for the product with V (half a step of each, against sum p |v|), and by what 32 bits do: the 128 products of a logit
    (an error of d in a logit is one of d in ln p; the fp32 sums of the tensor cores may truncate, a whole step of 2^-23 each) and the
    sums over the keys, joined in any order."""
    o64, l64, pv, sizes = ref
    u = HALF[dtype]
    d = 128 * 2.0 ** -23 * sizes + 2.0 ** -20
    acc = (n_keys + 64) * 2.0 ** -23
    tol = u * o64.abs() + (u * 1.01 + 2 * d[..., None] + 2 * acc) * pv + SMALL[dtype]
    err = (out.double() - o64).abs()
    assert torch.isfinite(out.double()).all(), f"{what}: outputs that are not finite"
    worst = (err / tol).max().item() if err.numel() else 0.0
    assert worst <= 1.0, f"{what}: an output is {worst:.2f} times its tolerance off (largest error {err.max().item():.3e})"
    if lse is not None:
        fin = torch.isfinite(l64)
        assert torch.equal(torch.isfinite(lse), fin), f"{what}: lse is infinite elsewhere"
        assert (lse[~fin] == -math.inf).all(), what
        tl = d + acc + 4 * 2.0 ** -23 * (l64.abs() + 16)
        e = (lse.double() - l64).abs()[fin] / tl[fin]
        assert e.numel() == 0 or e.max().item() <= 1.0, f"{what}: lse is {e.max().item():.2f} times its tolerance off"


def queries(T, Hq, dtype, seed, stride_extra=0):
    """[T, Hq, D], with `stride_extra` more heads between two tokens."""
    g = torch.Generator().manual_seed(seed + 1000)
    u = torch.randn((Hq + stride_extra, D), generator=g)
    x = (u + 0.5 * torch.randn((T, Hq + stride_extra, D), generator=g)).to(dtype).cuda()
    return x[:, :Hq]


def starts(lens):
    return torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], dtype=torch.int32, device="cuda")


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def workspace(p, n_tokens):
    n = cd.calidrop_paged_workspace_bytes(p, n_tokens)
    assert n > 0
    return torch.zeros((n,), dtype=torch.uint8, device="cuda")


def status_of(ws):
    torch.cuda.synchronize()
    return int(ws[:4].view(torch.int32).item())


def run_prefill(pool, q, q_lens, kv_lens, *, Hq, window=0, n_sink=0, pad=0, ws=None, scale=0.0, expect_status=0):
    T = q.shape[0]
    p = cd.make_paged_params(B=len(q_lens), Hq=Hq, Hkv=pool.Hkv, page_size=pool.page, n_pages=pool.n_pages, max_pages=pool.max_pages,
                             dtype=pool.dtype, window=window, n_sink=n_sink, softmax_scale=scale,
                             q_stride=q.stride(0) if T > 1 else 0, page_stride=pool.page_stride)
    ws = workspace(p, T) if ws is None else ws
    out = torch.full((T, Hq, D), 7.0, dtype=pool.dtype, device="cuda")
    lse = torch.full((T, Hq), 7.0, dtype=torch.float32, device="cuda")
    cd.calidrop_paged_prefill(p, q, pool.K, pool.V, pool.table, starts(q_lens), i32(kv_lens), out, lse, ws)
    assert status_of(ws) == expect_status
    return SimpleNamespace(p=p, out=out, lse=lse, ws=ws)


def check_prefill(pool, r, q, q_lens, kv_lens, *, Hq, window=0, n_sink=0, scale=None, prefix=None):
    """prefix: for each sequence (pool, index, length) of rows ahead of its own, or None."""
    G = Hq // pool.Hkv
    tok = 0
    scale = scale or 1.0 / math.sqrt(D)
    for b, (n, kv) in enumerate(zip(q_lens, kv_lens)):
        pos = torch.arange(kv - n, kv, device="cuda")
        for h in range(pool.Hkv):
            k, v = pool.k_rows[b][h, :kv], pool.v_rows[b][h, :kv]
            seen = visible(pos, kv, window, n_sink)
            if prefix and prefix[b]:
                pp, i, m = prefix[b]
                k, v = torch.cat([pp.k_rows[i][h, :m], k]), torch.cat([pp.v_rows[i][h, :m], v])
                seen = torch.cat([torch.ones((n, m), dtype=torch.bool, device="cuda"), seen], 1)
            for g in range(G):
                hq = h * G + g
                ref = attention64(q[tok:tok + n, hq], k, v, seen, scale)
                check_rows(r.out[tok:tok + n, hq], r.lse[tok:tok + n, hq], ref, pool.dtype, k.shape[0], f"sequence {b}, head {hq}")
        tok += n
    assert (r.out[tok:] == 7.0).all() and (r.lse[tok:] == 7.0).all(), "rows behind the last sequence were written"
