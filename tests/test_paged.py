"""The operators over a cache in pages, against their definitions in 64 bits."""
import math

import pytest
import torch

from paper_2507_19906_b200 import binding as cd
from paged_util import (D, HALF, SMALL, Pool, attention64, check_prefill, check_rows, i32, n_pages_of, queries, run_prefill, starts,
                        status_of, visible, workspace)

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


# ------------------------------------------------------------------------------------------ append
def table_of_angles(max_pos, rot):
    if not rot:
        return None
    a = torch.arange(max_pos, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)
    return torch.cat([a.cos(), a.sin()], 1).float().cuda()


def turned64(x, cs, rot, interleaved):
    """x [T, H, D] in 64 bits, and the sum of the terms' sizes for the tolerance."""
    y, size = x.double().clone(), x.double().abs()
    if rot:
        c, s = cs[:, None, :rot // 2].double(), cs[:, None, rot // 2:].double()
        i1 = torch.arange(0, rot, 2) if interleaved else torch.arange(rot // 2)
        i2 = i1 + (1 if interleaved else rot // 2)
        a, b = x[..., i1].double(), x[..., i2].double()
        y[..., i1], y[..., i2] = a * c - b * s, b * c + a * s
        size[..., i1] = (a * c).abs() + (b * s).abs()
        size[..., i2] = (b * c).abs() + (a * s).abs()
    return y, size


APPENDS = [
    # q_lens, old rows, Hq, Hkv, page, rot, interleaved, dtype, fused, positions, pad
    ([1], [0], 8, 8, 16, 128, False, BF, False, False, 0),
    ([1, 1, 1], [15, 16, 17], 32, 8, 16, 128, True, BF, False, False, 0),
    ([3, 0, 70, 1], [5, 9, 250, 0], 28, 4, 64, 64, False, FP, True, True, 2),
    ([0, 0, 130], [1, 2, 3], 12, 4, 128, 96, True, FP, True, False, 5),
    ([257, 2], [31, 600], 16, 2, 256, 32, False, BF, True, True, 0),
    ([1] * 70, list(range(70)), 24, 8, 32, 16, True, BF, False, False, 1),
    ([900, 33], [0, 100], 5, 1, 32, 0, False, BF, False, False, 3),
]


@pytest.mark.parametrize("case", APPENDS)
@pytest.mark.parametrize("with_q", [True, False])
def test_append(cuda_lib, case, with_q):
    q_lens, old, Hq, Hkv, page, rot, inter, dtype, fused, given, pad = case
    kv = [a + b for a, b in zip(q_lens, old)]
    pool = Pool(kv, Hkv=Hkv, page=page, dtype=dtype, interleaved_pool=fused)
    before_k, before_v = pool.K.clone(), pool.V.clone()
    T = sum(q_lens) + pad
    g = torch.Generator().manual_seed(3)
    if fused:
        x = torch.randn((T, Hq + 2 * Hkv, D), generator=g).to(dtype).cuda()
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    else:
        q, k, v = (torch.randn((T, n, D), generator=g).to(dtype).cuda() for n in (Hq, Hkv, Hkv))
    max_pos = max(kv) + 100
    cs = table_of_angles(max_pos, rot)
    place = torch.cat([torch.arange(o, o + n) for o, n in zip(old, q_lens)] + [torch.zeros(pad, dtype=torch.long)]).cuda()
    pos = torch.randint(0, max_pos, (T,), generator=g).int().cuda() if given else None
    p = cd.make_paged_params(B=len(kv), Hq=Hq, Hkv=Hkv, page_size=page, n_pages=pool.n_pages, max_pages=pool.max_pages, dtype=dtype,
                             rot_dim=rot, interleaved=inter, max_pos=max_pos, q_stride=q.stride(0) if fused else 0,
                             k_stride=k.stride(0) if fused else 0, v_stride=v.stride(0) if fused else 0, page_stride=pool.page_stride)
    ws = workspace(p, T)
    q_out = torch.full((T, Hq, D), 7.0, dtype=dtype, device="cuda")
    cd.calidrop_paged_append(p, q if with_q else None, k, v, pos, cs, pool.K, pool.V, pool.table, starts(q_lens), i32(kv), q_out, ws)
    assert status_of(ws) == 0
    n = T - pad
    angles = cs[(pos if given else place)[:n].long()] if rot else None
    u = HALF[dtype]
    got_k = torch.cat([pool.read(pool.K, b, kv[b])[:, old[b]:].transpose(0, 1) for b in range(len(kv))])
    got_v = torch.cat([pool.read(pool.V, b, kv[b])[:, old[b]:].transpose(0, 1) for b in range(len(kv))])
    assert torch.equal(got_v, v[:n])
    for got, x in [(got_k, k[:n])] + ([(q_out[:n], q[:n])] if with_q else []):
        ref, size = turned64(x, angles, rot, inter)
        # two products and a sum in 32 bits (each half a step of 2^-23), then the rounding
        tol = u * ref.abs() + 3 * 2.0 ** -24 * size + SMALL[dtype]
        assert ((got.double() - ref).abs() <= tol).all()
        assert torch.equal(got[..., rot:], x[..., rot:])
    assert (q_out[n if with_q else 0:] == 7.0).all()
    # nothing else of the pool has changed
    for b in range(len(kv)):
        pool.write(b, old[b], pool.k_rows[b][:, old[b]:], pool.v_rows[b][:, old[b]:])
    assert torch.equal(pool.K.view(torch.int16), before_k.view(torch.int16))
    assert torch.equal(pool.V.view(torch.int16), before_v.view(torch.int16))


def test_append_in_place_and_long_cache_offsets(cuda_lib):
    """q_out may be q; offsets into a pool of more than 2^31 elements."""
    Hq, Hkv, page = 16, 16, 256
    n_pages = (1 << 31) // (Hkv * page * D) + 8
    K = torch.zeros((n_pages, Hkv, page, D), dtype=BF, device="cuda")
    V = torch.zeros_like(K)
    g = torch.Generator().manual_seed(5)
    q, k, v = (torch.randn((2, 16, D), generator=g).to(BF).cuda() for _ in range(3))
    table = i32([[0, n_pages - 1], [1, n_pages - 2]])
    cs = table_of_angles(600, 128)
    p = cd.make_paged_params(B=2, Hq=Hq, Hkv=Hkv, page_size=page, n_pages=n_pages, max_pages=2, rot_dim=128, max_pos=600)
    ws = workspace(p, 2)
    kv = [512, 511]
    want, size = turned64(q, cs[[511, 510]], 128, False)
    wk, size_k = turned64(k, cs[[511, 510]], 128, False)
    cd.calidrop_paged_append(p, q, k, v, None, cs, K, V, table, i32([0, 1, 2]), i32(kv), q, ws)
    assert status_of(ws) == 0
    assert ((q.double() - want).abs() <= 2.0 ** -8 * want.abs() + 3 * 2.0 ** -24 * size).all()
    for b in range(2):
        pg, row = n_pages - 1 - b, (kv[b] - 1) % page
        assert torch.equal(V[pg, :, row], v[b])
        assert ((K[pg, :, row].double() - wk[b]).abs() <= 2.0 ** -8 * wk[b].abs() + 3 * 2.0 ** -24 * size_k[b]).all()
    # and attention reads them: only the last rows have logits that are not zero
    out = torch.empty_like(q)
    lse = torch.empty((2, Hq), device="cuda")
    cd.calidrop_paged_decode(p, q, K, V, table, i32(kv), out, lse, ws)
    out2, lse2 = torch.empty_like(q), torch.empty_like(lse)
    cd.calidrop_paged_prefill(p, q, K, V, table, i32([0, 1, 2]), i32(kv), out2, lse2, ws)
    assert status_of(ws) == 0
    for b in range(2):
        for h in range(Hkv):
            kk = torch.zeros((kv[b], D), dtype=BF, device="cuda")
            vv = torch.zeros_like(kk)
            kk[-1], vv[-1] = K[n_pages - 1 - b, h, (kv[b] - 1) % page], v[b, h]
            ref = attention64(q[b:b + 1, h], kk, vv, torch.ones((1, kv[b]), dtype=torch.bool, device="cuda"), 1 / math.sqrt(D))
            check_rows(out[b:b + 1, h], lse[b:b + 1, h], ref, BF, kv[b])
            check_rows(out2[b:b + 1, h], lse2[b:b + 1, h], ref, BF, kv[b])


# ------------------------------------------------------------------------------------------ decode
DECODES = [
    # kv_lens, Hq, Hkv, page, window, sink, dtype
    ([1], 8, 8, 16, 0, 0, BF),
    ([0, 1, 2], 32, 8, 64, 0, 0, BF),
    ([63, 64, 65, 128, 129], 28, 4, 16, 0, 0, FP),
    ([700], 5, 1, 128, 0, 0, BF),
    ([3000, 17, 0, 999], 24, 8, 32, 0, 0, FP),
    ([20000], 16, 2, 256, 0, 0, BF),
    ([2111], 32, 8, 64, 480, 32, BF),
    ([500, 40, 1000, 33], 32, 32, 16, 100, 5, BF),
    ([777, 130, 64], 12, 4, 64, 1, 0, FP),
    ([777, 130, 64], 12, 4, 32, 1, 200, BF),
    ([5000, 1], 40, 8, 128, 65, 1, BF),
    ([900], 8, 1, 64, 1000, 3, BF),
    (list(range(300, 340)), 14, 2, 64, 64, 64, FP),
]


def run_decode(pool, q, kv, *, Hq, window=0, n_sink=0, ws=None, expect_status=0):
    B = len(kv)
    p = cd.make_paged_params(B=B, Hq=Hq, Hkv=pool.Hkv, page_size=pool.page, n_pages=pool.n_pages, max_pages=pool.max_pages, dtype=pool.dtype,
                             window=window, n_sink=n_sink, q_stride=q.stride(0) if B > 1 else 0, page_stride=pool.page_stride)
    ws = workspace(p, B) if ws is None else ws
    r = type("R", (), {})()
    r.out = torch.full((B, Hq, D), 7.0, dtype=pool.dtype, device="cuda")
    r.lse = torch.full((B, Hq), 7.0, device="cuda")
    r.ws, r.p = ws, p
    cd.calidrop_paged_decode(p, q, pool.K, pool.V, pool.table, i32(kv), r.out, r.lse, ws)
    assert status_of(ws) == expect_status
    return r


@pytest.mark.parametrize("case", DECODES)
def test_decode(cuda_lib, case):
    kv, Hq, Hkv, page, window, sink, dtype = case
    pool = Pool(kv, Hkv=Hkv, page=page, dtype=dtype, seed=len(kv), interleaved_pool=page == 64)
    for b in range(len(kv)):
        if window:
            pool.hide(b, window, sink, kv[b] - 1)
    q = queries(len(kv), Hq, dtype, 1, stride_extra=4 if page == 32 else 0)
    r = run_decode(pool, q, kv, Hq=Hq, window=window, n_sink=sink)
    check_prefill(pool, r, q, [1] * len(kv), kv, Hq=Hq, window=window, n_sink=sink)
    # again in the same workspace: it was left ready
    r2 = run_decode(pool, q, kv, Hq=Hq, window=window, n_sink=sink, ws=r.ws)
    assert torch.equal(r.out, r2.out) and torch.equal(r.lse, r2.lse)


def test_decode_of_many_sequences(cuda_lib):
    """More sequences than threads of a CTA, most of them tiny."""
    kv = [(i * 37) % 90 for i in range(700)] + [3000]
    pool = Pool(kv, Hkv=2, page=16, seed=4)
    q = queries(len(kv), 8, BF, 2)
    r = run_decode(pool, q, kv, Hq=8, window=70, n_sink=3)
    check_prefill(pool, r, q, [1] * len(kv), kv, Hq=8, window=70, n_sink=3)


# ------------------------------------------------------------------------------------------ prefill
PREFILLS = [
    # q_lens, kv_lens, Hq, Hkv, page, window, sink, dtype, pad
    ([1], [1], 8, 8, 16, 0, 0, BF, 0),
    ([128], [128], 8, 8, 128, 0, 0, BF, 0),
    ([129], [129], 2, 2, 64, 0, 0, FP, 0),
    ([300], [300], 32, 8, 64, 0, 0, BF, 0),
    ([5, 0, 1, 300], [5, 0, 700, 300], 28, 4, 16, 0, 0, FP, 3),
    ([10, 3, 2], [4, 0, 2], 12, 4, 32, 0, 0, BF, 1),
    ([64, 65], [1000, 2000], 40, 8, 256, 0, 0, BF, 0),
    ([3], [5000], 16, 2, 64, 0, 0, BF, 0),
    ([257], [257], 5, 1, 128, 0, 0, BF, 0),
    ([513], [513], 8, 1, 64, 0, 0, FP, 0),
    ([700], [700], 32, 8, 64, 100, 5, BF, 0),
    ([400, 33], [900, 40], 24, 8, 16, 64, 0, FP, 2),
    ([600], [600], 6, 2, 32, 1, 0, BF, 0),
    ([600], [600], 6, 2, 32, 1, 300, BF, 0),
    ([150], [3000], 16, 2, 128, 700, 130, BF, 0),
    ([1, 1, 1, 1], [50, 600, 1000, 1], 32, 8, 64, 256, 32, BF, 0),
    ([1000], [1100], 4, 4, 64, 128, 128, FP, 0),
    # more tiles of rows than a warp lists, some of them cut along the keys
    ([3000], [3000], 8, 2, 64, 0, 0, BF, 0),
    # more sequences than a warp counts, some with most of the work
    ([1, 0, 3, 40] * 12 + [300, 130], [5, 0, 700, 40] * 12 + [2500, 130], 8, 2, 16, 0, 0, FP, 1),
    # more sequences than a CTA has threads
    ([1] * 650 + [70], [1 + i % 130 for i in range(650)] + [1500], 4, 1, 16, 90, 4, BF, 0),
]


@pytest.mark.parametrize("case", PREFILLS)
def test_prefill(cuda_lib, case):
    q_lens, kv, Hq, Hkv, page, window, sink, dtype, pad = case
    pool = Pool(kv, Hkv=Hkv, page=page, dtype=dtype, seed=len(kv), interleaved_pool=page == 64)
    if window:
        for b in range(len(kv)):
            pool.hide(b, window, sink, kv[b] - q_lens[b])
    q = queries(sum(q_lens) + pad, Hq, dtype, 1, stride_extra=4 if page == 32 else 0)
    r = run_prefill(pool, q, q_lens, kv, Hq=Hq, window=window, n_sink=sink)
    check_prefill(pool, r, q, q_lens, kv, Hq=Hq, window=window, n_sink=sink)
    r2 = run_prefill(pool, q, q_lens, kv, Hq=Hq, window=window, n_sink=sink, ws=r.ws)
    assert torch.equal(r.out, r2.out) and torch.equal(r.lse, r2.lse)


def test_prefill_rescales_and_takes_large_logits(cuda_lib):
    """Maxima that grow from tile to tile by more than the lazy rescaling leaves, and rows that differ in it; a scale of the caller's."""
    n = 1024
    pool = Pool([n], Hkv=2, page=64, seed=2)
    ramp = torch.linspace(0.0, 40.0, n)[None, :, None]
    u = torch.randn(D, generator=torch.Generator().manual_seed(1))
    pool.k_rows[0] = (pool.k_rows[0].cpu().float() + ramp * u / u.norm()).to(BF).cuda()
    pool.write(0, 0, pool.k_rows[0], pool.v_rows[0])
    q = queries(n, 8, BF, 3)
    q = (q.float() + (torch.arange(n, device="cuda") % 5 == 0)[:, None, None] * 4.0 * u.cuda()).to(BF)
    for scale in (0.0, 0.3):
        r = run_prefill(pool, q, [n], [n], Hq=8, scale=scale)
        check_prefill(pool, r, q, [n], [n], Hq=8, scale=scale or None)


# ------------------------------------------------------------------------------------------ shared prefix
PREFIXES = [
    # members of the groups (the last: of no group), prefix lengths, own lengths' pattern, Hq, Hkv, page, dtype
    ([1, 0], [1], 1, 8, 8, 16, BF),
    ([8, 0], [1000], 65, 32, 8, 64, BF),
    ([3, 5, 0], [300, 0], 20, 28, 4, 32, FP),
    ([70, 0], [513], 9, 32, 8, 64, BF),
    ([2, 1, 4, 3], [64, 2000, 129], 40, 16, 2, 128, FP),
    ([33, 0], [4000], 0, 40, 8, 256, BF),
    ([0, 9, 2], [100, 700], 130, 5, 1, 16, BF),
    # more groups than a warp counts, one with most of the rows
    ([2, 1, 0, 3] * 10 + [1], [17 * i % 200 for i in range(39)] + [3000], 10, 8, 2, 32, BF),
]


@pytest.mark.parametrize("case", PREFIXES)
def test_prefix_decode(cuda_lib, case):
    members, plens, own, Hq, Hkv, page, dtype = case
    B, n_groups = sum(members), len(plens)
    kv = [(i * 13) % (own + 1) for i in range(B)]
    both = Pool(kv + plens, Hkv=Hkv, page=page, dtype=dtype, seed=B, interleaved_pool=page == 32)
    table, prefix_table = both.table[:B].contiguous(), both.table[B:].contiguous()
    q = queries(B, Hq, dtype, 1, stride_extra=4 if page == 32 else 0)
    borders = [sum(members[:i]) for i in range(n_groups + 1)]
    p = cd.make_paged_params(B=B, Hq=Hq, Hkv=Hkv, page_size=page, n_pages=both.n_pages, max_pages=both.max_pages, dtype=dtype,
                             n_groups=n_groups, max_prefix_pages=both.max_pages, q_stride=q.stride(0) if B > 1 else 0,
                             page_stride=both.page_stride)
    ws = workspace(p, B)
    prefix = []
    for g, n in enumerate(members):
        prefix += [(both, B + g, plens[g]) if g < n_groups else None] * n
    for _ in range(2):
        r = type("R", (), {})()
        r.out = torch.full((B, Hq, D), 7.0, dtype=dtype, device="cuda")
        r.lse = torch.full((B, Hq), 7.0, device="cuda")
        cd.calidrop_paged_prefix_decode(p, q, both.K, both.V, i32(borders), prefix_table, i32(plens), table, i32(kv), r.out, r.lse, ws)
        assert status_of(ws) == 0
        check_prefill(both, r, q, [1] * B, kv, Hq=Hq, prefix=prefix)


def test_no_tokens(cuda_lib):
    pool = Pool([100], Hkv=2, page=64)
    p = cd.make_paged_params(B=1, Hq=8, Hkv=2, page_size=64, n_pages=pool.n_pages, max_pages=pool.max_pages)
    ws = workspace(p, 0)
    q = torch.empty((0, 8, D), dtype=BF, device="cuda")
    k = torch.empty((0, 2, D), dtype=BF, device="cuda")
    z = i32([0, 0])
    n = cd.calidrop_launch_count()
    cd.calidrop_paged_prefill(p, q, pool.K, pool.V, pool.table, z, i32([100]), q, None, ws)
    cd.calidrop_paged_append(p, q, k, k, None, None, pool.K, pool.V, pool.table, z, i32([100]), q, ws)
    assert cd.calidrop_launch_count() == n and status_of(ws) == 0
    # tokens that are all padding
    q = queries(5, 8, BF, 1)
    r = run_prefill(pool, q, [0], [100], Hq=8)
    check_prefill(pool, r, q, [0], [100], Hq=8)


def test_calls_at_once(cuda_lib):
    """Two streams with a workspace each, over the same cache; and calls of every kind in turn in one workspace."""
    kv = [900, 30, 2000]
    pool = Pool(kv, Hkv=2, page=32, seed=3)
    q = queries(3 + 200, 8, BF, 4)
    p = cd.make_paged_params(B=3, Hq=8, Hkv=2, page_size=32, n_pages=pool.n_pages, max_pages=pool.max_pages, n_groups=1,
                             max_prefix_pages=pool.max_pages)
    lens, new = i32(kv), [100, 3, 100]
    st = starts(new)
    out = {}
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for round_ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                if round_ == 0:
                    out[i] = dict(ws=workspace(p, 203), o=[torch.empty_like(q) for _ in range(3)], l=[torch.empty((203, 8), device="cuda") for _ in range(3)])
                w = out[i]
                cd.calidrop_paged_prefill(p, q, pool.K, pool.V, pool.table, st, lens, w["o"][0], w["l"][0], w["ws"])
                cd.calidrop_paged_decode(p, q[:3], pool.K, pool.V, pool.table, lens, w["o"][1][:3], w["l"][1][:3], w["ws"])
                cd.calidrop_paged_prefix_decode(p, q[:3], pool.K, pool.V, i32([0, 2]), pool.table[2:], lens[2:], pool.table, lens, w["o"][2][:3],
                                                w["l"][2][:3], w["ws"])
    torch.cuda.synchronize()
    for w in out.values():
        assert status_of(w["ws"]) == 0
        r = type("R", (), {})
        r.out, r.lse = w["o"][0], w["l"][0]
        check_prefill(pool, r, q, new, kv, Hq=8)
        r.out, r.lse = w["o"][1][:3], w["l"][1][:3]
        check_prefill(pool, r, q[:3], [1] * 3, kv, Hq=8)
        r.out, r.lse = w["o"][2][:3], w["l"][2][:3]
        check_prefill(pool, r, q[:3], [1] * 3, kv, Hq=8, prefix=[(pool, 2, kv[2]), (pool, 2, kv[2]), None])


# ------------------------------------------------------------------------------------------ masked and broken data
def test_infinite_values_where_nothing_is_seen(cuda_lib):
    """K and V of rows outside the window, behind the length and in other pages hold infinities and NaN: no effect."""
    kv, W, sink = 500, 70, 3
    for bad in (math.inf, -math.inf, math.nan):
        pool = Pool([kv], Hkv=2, page=64, seed=1)
        hidden = [t for t in range(kv) if sink <= t <= kv - 1 - W]
        for x in (pool.K, pool.V):
            for t in hidden:
                x[pool.table[0, t // 64].long(), :, t % 64] = bad
        q = queries(1, 8, BF, 2)
        r = run_decode(pool, q, [kv], Hq=8, window=W, n_sink=sink)
        check_prefill(pool, r, q, [1], [kv], Hq=8, window=W, n_sink=sink)
        r = run_prefill(pool, q, [1], [kv], Hq=8, window=W, n_sink=sink)
        check_prefill(pool, r, q, [1], [kv], Hq=8, window=W, n_sink=sink)


def test_keys_that_are_not_finite_stay_with_those_who_see_them(cuda_lib):
    """A NaN key makes NaN of the tokens that see it and of no others; a key at minus infinity drops out."""
    n = 300
    pool = Pool([n], Hkv=2, page=64, seed=1)
    k0 = pool.k_rows[0].clone()
    q = queries(n, 8, BF, 2)
    pool.k_rows[0] = k0.clone()
    pool.k_rows[0][:, 200] = math.nan
    pool.write(0, 0, pool.k_rows[0], pool.v_rows[0])
    r = run_prefill(pool, q, [n], [n], Hq=8)
    assert torch.isnan(r.out[200:].float()).all() and torch.isnan(r.lse[200:]).all()
    pool.k_rows[0] = k0
    early = type("R", (), dict(out=r.out[:200], lse=r.lse[:200]))
    check_prefill(pool, early, q[:200], [200], [200], Hq=8)


@pytest.mark.parametrize("what", ["page", "low page", "long", "negative", "position"])
def test_bad_device_data_is_flagged(cuda_lib, what):
    kv = [200, 300]
    pool = Pool(kv, Hkv=2, page=64, seed=1)
    q = queries(2, 8, BF, 2)
    good = run_decode(pool, q, kv, Hq=8)
    lens, bit = list(kv), 1
    pos = None
    if what == "page":
        pool.table[0, 1], bit = pool.n_pages, 2
    elif what == "low page":
        pool.table[0, 1], bit = -1, 2
    elif what == "long":
        lens[0] = pool.max_pages * 64 + 1
    elif what == "negative":
        lens[0] = -1
    else:
        pos, bit = i32([5, 1000]), 4
    cs = table_of_angles(400, 128)
    p = cd.make_paged_params(B=2, Hq=8, Hkv=2, page_size=64, n_pages=pool.n_pages, max_pages=pool.max_pages, rot_dim=128, max_pos=400)
    if what != "position":
        if what == "long":
            pool.table[0, 4:] = pool.table[1, 4]    # a page that exists
        for run in (lambda: run_decode(pool, q, lens, Hq=8, expect_status=bit), lambda: run_prefill(pool, q, [1, 1], lens, Hq=8, expect_status=bit)):
            r = run()
            assert torch.allclose(r.out[1].float(), good.out[1].float(), atol=2e-2)      # the other sequence's are right
    ws = workspace(p, 2)
    K, V = pool.K.clone(), pool.V.clone()
    k = torch.randn((2, 2, D), device="cuda").to(BF)
    at = list(lens)
    if what in ("page", "low page"):
        at[0] = 100                                                                       # a token whose page is the bad one
    cd.calidrop_paged_append(p, None, k, k, pos, cs, K, V, pool.table, i32([0, 1, 2]), i32(at), None, ws)
    assert status_of(ws) == bit
    row = (K.view(torch.int16) != pool.K.view(torch.int16)).any(-1)
    assert row.sum().item() == 2                                                          # one token's rows: two heads


def test_falling_starts_are_flagged(cuda_lib):
    pool = Pool([200, 300, 100], Hkv=2, page=64, seed=1)
    p = cd.make_paged_params(B=3, Hq=8, Hkv=2, page_size=64, n_pages=pool.n_pages, max_pages=pool.max_pages)
    q = queries(40, 8, BF, 2)
    for s in ([0, 30, 10, 40], [0, 10, 20, 41], [-1, 10, 20, 40], [0, 1 << 30, -(1 << 30), 40]):
        ws = workspace(p, 40)
        out = torch.empty_like(q)
        cd.calidrop_paged_prefill(p, q, pool.K, pool.V, pool.table, i32(s), i32([200, 300, 100]), out, None, ws)
        assert status_of(ws) & 1 and status_of(ws) < 8


# ------------------------------------------------------------------------------------------ streams, graphs, and a run of them together
def test_captured_calls_follow_the_lengths(cuda_lib):
    """A captured decode step, replayed after the lengths and the table have changed, on a stream of its own; two graphs, a workspace each."""
    B, Hq, Hkv = 3, 8, 2
    pool = Pool([700, 500, 900], Hkv=Hkv, page=64, seed=1)
    q = queries(B, Hq, BF, 2)
    p = cd.make_paged_params(B=B, Hq=Hq, Hkv=Hkv, page_size=64, n_pages=pool.n_pages, max_pages=pool.max_pages, window=300, n_sink=4)
    graphs, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    kv = i32([1, 1, 1])
    for s in streams:
        ws, out, lse = workspace(p, B), torch.empty_like(q), torch.empty((B, Hq), device="cuda")
        out2, lse2 = torch.empty_like(q), torch.empty((B, Hq), device="cuda")
        st = starts([1] * B)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            cd.calidrop_paged_decode(p, q, pool.K, pool.V, pool.table, kv, out, lse, ws)
            s.synchronize()
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                cd.calidrop_paged_decode(p, q, pool.K, pool.V, pool.table, kv, out, lse, ws)
                cd.calidrop_paged_prefill(p, q, pool.K, pool.V, pool.table, st, kv, out2, lse2, ws)
        graphs.append((g, s, ws, out, lse, out2, lse2, st))
    for lens in ([700, 500, 900], [64, 0, 65], [333, 499, 1]):
        kv.copy_(i32(lens))
        torch.cuda.synchronize()
        for g, s, *_ in graphs:
            with torch.cuda.stream(s):
                g.replay()
        for g, s, ws, out, lse, out2, lse2, st in graphs:
            assert status_of(ws) == 0
            check_prefill(pool, type("R", (), dict(out=out, lse=lse)), q, [1] * B, lens, Hq=Hq, window=300, n_sink=4)
            check_prefill(pool, type("R", (), dict(out=out2, lse=lse2)), q, [1] * B, lens, Hq=Hq, window=300, n_sink=4)


def test_window_with_sinks_is_the_streaming_rule(cuda_lib):
    """The mask over the whole cache gives what calidrop_decode gives over the cache that calidrop_select_streaming keeps."""
    B, Hq, Hkv, L, budget, sink = 2, 8, 2, 900, 200, 32
    pool = Pool([L] * B, Hkv=Hkv, page=64, seed=1)
    q = queries(B, Hq, BF, 2)
    r = run_decode(pool, q, [L] * B, Hq=Hq, window=budget - sink, n_sink=sink)
    p = cd.make_params(B=B, Hq=Hq, Hkv=Hkv, L=L, window=1, budget=budget, cap=budget, n_cal=1, theta2=2.0)
    K, V = torch.stack(pool.k_rows), torch.stack(pool.v_rows)
    st = cd.alloc_layer_state(p)
    cd.calidrop_select_streaming(p, sink, st.kept_idx)
    cd.calidrop_calibrate(p, q[:, :, None].contiguous(), K, V, None, st.kept_idx, st.K_kept, st.V_kept, st.O_c, st.LSE_c, st.C_q, st.ws_compress)
    out, lse = torch.empty_like(q), torch.empty((B, Hq), device="cuda")
    cd.calidrop_decode(p, q, None, None, st.K_kept, st.V_kept, budget, st.O_c, st.LSE_c, st.C_q, out, lse, None, st.ws_decode)
    torch.cuda.synchronize()
    assert (out.float() - r.out.float()).abs().max().item() <= 2e-2
    assert (lse - r.lse).abs().max().item() <= 1e-4


def test_a_serving_run(cuda_lib):
    """Prompts appended and prefilled in chunks, their row LSE handed to calidrop_compress, then tokens appended and decoded, with and
    without the prompt as a shared prefix."""
    Hq, Hkv, page, W = 8, 2, 64, 16
    G = Hq // Hkv
    B, prompt, steps = 2, [500, 333], 3
    total = [n + steps for n in prompt]
    g = torch.Generator().manual_seed(11)
    raw = [[torch.randn((n, h, D), generator=g).to(BF).cuda() for h in (Hq, Hkv, Hkv)] for n in total]
    cs = table_of_angles(600, 128)
    pool = Pool(total, Hkv=Hkv, page=page, seed=3)
    pool.K.fill_(math.nan)
    pool.V.fill_(math.nan)
    p = cd.make_paged_params(B=B, Hq=Hq, Hkv=Hkv, page_size=page, n_pages=pool.n_pages, max_pages=pool.max_pages, rot_dim=128, max_pos=600)
    ws = workspace(p, 600)

    def exactly(n0, n1, b):            # rotated in 64 bits, rounded once
        at = torch.arange(n0, n1)
        return [turned64(raw[b][i][n0:n1], cs[at], 128, False)[0].to(BF) for i in (0, 1)]

    def step(lens, new):
        q, k, v = (torch.cat([raw[b][i][lens[b] - new[b]:lens[b]] for b in range(B)]) for i in range(3))
        qr = torch.empty_like(q)
        cd.calidrop_paged_append(p, q, k, v, None, cs, pool.K, pool.V, pool.table, starts(new), i32(lens), qr, ws)
        return qr

    def cached(lens):
        for b in range(B):
            k = exactly(0, lens[b], b)[1].transpose(0, 1)
            got = pool.read(pool.K, b, lens[b])
            # an fp32 rotation may round the other way than one in 64 bits: a whole step
            assert ((got.float() - k.float()).abs() <= 2 * HALF[BF] * k.float().abs() + 1e-6).all()
            pool.k_rows[b], pool.v_rows[b] = got, raw[b][2][:lens[b]].transpose(0, 1)

    lens = [0, 0]
    keep = None
    for new in ([200, 333], [300, 0]):
        lens = [a + b for a, b in zip(lens, new)]
        qr = step(lens, new)
        out, lse = torch.empty_like(qr), torch.empty((sum(new), Hq), device="cuda")
        cd.calidrop_paged_prefill(p, qr, pool.K, pool.V, pool.table, starts(new), i32(lens), out, lse, ws)
        assert status_of(ws) == 0
        cached(lens)
        check_prefill(pool, type("R", (), dict(out=out, lse=lse)), qr, new, lens, Hq=Hq)
        keep = qr, lse
    # sequence 0's window rows: its LSE is what the compression's own statistics pass finds
    qr, lse = keep
    L = prompt[0]
    cp = cd.make_params(B=1, Hq=Hq, Hkv=Hkv, L=L, window=W, pool=5, budget=100, n_cal=W, cap=100)
    Q_obs = qr[-W:].transpose(0, 1).contiguous()[None]
    K, V = (pool.read(x, 0, L).contiguous()[None] for x in (pool.K, pool.V))
    st = [cd.alloc_layer_state(cp) for _ in range(2)]
    for s, obs in zip(st, (None, lse[-W:].t().contiguous()[None])):
        cd.calidrop_compress(cp, Q_obs, K, V, obs, s.kept_idx, s.K_kept, s.V_kept, s.O_c, s.LSE_c, s.C_q, s.ws_compress)
    torch.cuda.synchronize()
    assert torch.equal(st[0].kept_idx, st[1].kept_idx)
    assert (st[0].LSE_c - st[1].LSE_c).abs().max().item() <= 1e-3
    assert (st[0].O_c - st[1].O_c).abs().max().item() <= 2e-2
    # tokens
    for t in range(steps):
        lens = [n + 1 for n in lens]
        qr = step(lens, [1, 1])
        out, lse = torch.empty_like(qr), torch.empty((B, Hq), device="cuda")
        cd.calidrop_paged_decode(p, qr, pool.K, pool.V, pool.table, i32(lens), out, lse, ws)
        assert status_of(ws) == 0
        cached(lens)
        check_prefill(pool, type("R", (), dict(out=out, lse=lse)), qr, [1, 1], lens, Hq=Hq)
    # both sequences as two readers of sequence 0's prompt, with what follows it as their own rows
    n_pre = 448                                        # whole pages: the rest of sequence 0 is its own
    pp = cd.make_paged_params(B=1, Hq=Hq, Hkv=Hkv, page_size=page, n_pages=pool.n_pages, max_pages=1, n_groups=1, max_prefix_pages=7)
    ws2 = workspace(pp, 1)
    o2, l2 = torch.empty_like(out[:1]), torch.empty_like(lse[:1])
    cd.calidrop_paged_prefix_decode(pp, qr[:1].contiguous(), pool.K, pool.V, i32([0, 1]), pool.table[:1, :7].contiguous(), i32([n_pre]),
                                    pool.table[:1, 7:8].contiguous(), i32([lens[0] - n_pre]), o2, l2, ws2)
    assert status_of(ws2) == 0
    check_prefill(pool, type("R", (), dict(out=o2, lse=l2)), qr[:1], [1], lens[:1], Hq=Hq)
