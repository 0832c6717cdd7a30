"""Bad and extreme device data in the operators over a cache in pages: what is flagged, what stays right beside it."""
import math

import pytest
import torch

from paper_2507_19906_b200 import binding as cd
from paged_util import (D, HALF, SMALL, Pool, attention64, check_prefill, check_rows, i32, queries, run_prefill, starts, status_of,
                        workspace)
from test_paged import table_of_angles, turned64

pytestmark = pytest.mark.gpu

BF, FP = torch.bfloat16, torch.float16


# ------------------------------------------------------------------------------------------ shared prefix
class Prefixed:
    """B sequences of a few own rows, and prefixes for `plens` groups, in one pool."""

    def __init__(self, B, plens, own, Hq=8, Hkv=2, page=32, dtype=BF):
        self.B, self.plens, self.Hq = B, plens, Hq
        self.kv = [1 + (i * 13) % own for i in range(B)]
        self.pool = Pool(self.kv + plens, Hkv=Hkv, page=page, dtype=dtype, seed=B)
        self.table, self.prefix_table = self.pool.table[:B].contiguous(), self.pool.table[B:].contiguous()
        self.q = queries(B, Hq, dtype, 1)
        self.p = cd.make_paged_params(B=B, Hq=Hq, Hkv=Hkv, page_size=page, n_pages=self.pool.n_pages, max_pages=self.pool.max_pages, dtype=dtype,
                                      n_groups=len(plens), max_prefix_pages=self.pool.max_pages)
        self.ws = workspace(self.p, B)
        # where a call with groups keeps, for each token, which partial rows are its own: 16 bytes each, behind the parts whose size
        # depends on nothing
        none = cd.make_paged_params(B=B, Hq=Hq, Hkv=Hkv, page_size=page, n_pages=self.pool.n_pages, max_pages=self.pool.max_pages, dtype=dtype)
        at = cd.calidrop_paged_workspace_bytes(none, 0)
        self.records = self.ws[at:at + 16 * B].view(torch.int32)

    def run(self, borders, plens=None, kv=None):
        r = type("R", (), {})()
        r.out = torch.full_like(self.q, 7.0)
        r.lse = torch.full((self.B, self.Hq), 7.0, device="cuda")
        cd.calidrop_paged_prefix_decode(self.p, self.q, self.pool.K, self.pool.V, i32(borders), self.prefix_table, i32(plens or self.plens),
                                        self.table, i32(kv or self.kv), r.out, r.lse, self.ws)
        r.status = status_of(self.ws)
        self.ws[:4].zero_()
        return r

    def check(self, r, b, prefix):
        """Sequence b, over the prefix of that index (None: its own rows only)."""
        one = type("R", (), dict(out=r.out[b:b + 1], lse=r.lse[b:b + 1]))
        pool = self.pool
        rows = type("P", (), dict(Hkv=pool.Hkv, dtype=pool.dtype, k_rows=[pool.k_rows[b]], v_rows=[pool.v_rows[b]]))
        check_prefill(rows, one, self.q[b:b + 1], [1], [self.kv[b]], Hq=self.Hq,
                      prefix=None if prefix is None else [(pool, self.B + prefix, self.plens[prefix])])


@pytest.mark.parametrize("n_groups", [3, 40])
def test_prefix_groups_that_are_not_taken(cuda_lib, n_groups):
    """A group_start that passes B, falls or is negative is flagged; the sequences of those groups have their own rows only, whatever
    an earlier call left in the workspace, and the other groups' are right."""
    x = Prefixed(90, [200 + 10 * (g % 3) for g in range(n_groups)], 40)
    base = [0, 30, 60, 90] if n_groups == 3 else [2 * g for g in range(n_groups)] + [90]
    for change in ({}, {2: 91}, {1: -1}, {0: -5}, {n_groups: 1 << 30}, {1: 70} if n_groups == 3 else {1: 5}):
        borders = list(base)
        for i, v in change.items():
            borders[i] = v
        # what a call without groups may have left there: a row whose maximum is 0 and whose sum is 1.0, 1.0, ...
        x.records.copy_(i32([0, 0x3f800000, 0, 0] * x.B))
        r = x.run(borders)
        assert r.status == (1 if change else 0), (change, r.status)
        taken = [g for g in range(n_groups) if 0 <= borders[g] <= borders[g + 1] <= x.B]
        for b in range(x.B):
            of = [g for g in taken if borders[g] <= b < borders[g + 1]]
            if len(of) <= 1:              # (a start that falls puts sequences into two groups: undefined)
                x.check(r, b, of[0] if of else None)


@pytest.mark.parametrize("n_groups", [5, 41])
def test_prefix_groups_that_lie_over_one_another(cuda_lib, n_groups):
    """Starts that fall all the time, between groups that are each good: flagged.  With more groups than a warp counts, their tiles are
    more than starts that do not fall could have: the list of work is given up, and all sequences have their own rows only."""
    x = Prefixed(96, [200] * n_groups, 40, Hq=16, Hkv=2)
    borders = [0, 96] * (n_groups // 2 + 1)
    for _ in range(3):
        x.records.copy_(i32([0, 0x3f800000, 0, 0] * x.B))
        r = x.run(borders[:n_groups + 1])
        assert r.status == 1
        if n_groups > 32:
            for b in (0, 1, 50, 95):
                x.check(r, b, None)
    r = x.run([0] * n_groups + [96])               # and the same workspace is ready for starts that do not fall
    assert r.status == 0
    for b in (0, 1, 50, 95):
        x.check(r, b, n_groups - 1)


# ------------------------------------------------------------------------------------------ append
class Appended:
    """A batch in pages whose rows are all there, and new tokens for it."""

    def __init__(self, kv, T, Hkv=2, page=64, spare=3):
        self.kv, self.T, self.Hkv = kv, T, Hkv
        self.pool = Pool(kv, Hkv=Hkv, page=page, seed=1, spare=spare)
        self.p = cd.make_paged_params(B=len(kv), Hq=8, Hkv=Hkv, page_size=page, n_pages=self.pool.n_pages, max_pages=self.pool.max_pages)
        g = torch.Generator().manual_seed(7)
        self.q, self.k, self.v = (torch.randn((T, h, D), generator=g).to(BF).cuda() for h in (8, Hkv, Hkv))

    def run(self, q_start, kv=None):
        """The status, and which tokens were stored (anywhere), by their keys."""
        K, V = self.pool.K.clone(), self.pool.V.clone()
        ws, q_out = workspace(self.p, self.T), torch.full_like(self.q, 7.0)
        cd.calidrop_paged_append(self.p, self.q, self.k, self.v, None, None, K, V, self.pool.table, i32(q_start), i32(kv or self.kv), q_out, ws)
        status = status_of(ws)
        rows = K.transpose(1, 2).reshape(-1, self.Hkv * D).view(torch.int16)
        old = self.pool.K.transpose(1, 2).reshape(-1, self.Hkv * D).view(torch.int16)
        changed = rows[(rows != old).any(1)]
        keys = self.k.reshape(self.T, -1).view(torch.int16)
        stored = (changed[:, None] == keys[None]).all(2).any(0) if len(changed) else torch.zeros(self.T, dtype=torch.bool, device="cuda")
        assert (changed[:, None] == keys[None]).all(2).any(1).all(), "a row is no token's"
        assert torch.equal((q_out != 7.0).flatten(1).any(1), stored)
        return status, stored.tolist()


@pytest.mark.parametrize("starts,taken", [
    ([0, 10, 20, 40], range(40)),
    ([0, 10, 20, 35], range(35)),                 # what lies behind is padding
    ([0, 10, 20, 41], range(20)),                 # passes the tokens
    ([0, 10, 20, 1 << 30], range(20)),
    ([0, 30, 10, 40], None),                      # falls
    ([0, 20, 30, 10], None),                      # falls at the end: all tokens behind it are padding
    ([0, 20, 30, -1], ()),
    ([-1, 10, 20, 40], None),
    ([5, 5, 20, 40], None),
    ([0, 1 << 30, -(1 << 30), 40], None),
    ([41, 41, 41, 41], ()),
    ([-3, -2, -1, 0], ()),
])
def test_append_starts(cuda_lib, starts, taken):
    """The starts that calidrop_paged_prefill flags are flagged by the append, too, and the tokens of sequences that pass the end are left out."""
    x = Appended([200, 300, 100], 40)
    status, stored = x.run(starts)
    good = all(0 <= a <= b <= 40 for a, b in zip(starts, starts[1:])) and starts[0] in (0, 41)
    assert status == (0 if good else 1)
    if taken is not None:
        assert [t for t in range(40) if stored[t]] == list(taken)


def test_append_starts_of_many_sequences(cuda_lib):
    """One bad start among more sequences than a block has threads, without tokens."""
    B = 700
    x = Appended([5] * B, 3, spare=0)
    base = [0] * 600 + [3] * (B + 1 - 600)
    assert x.run(base, [5] * B)[0] == 0
    for at, v in ((300, 4), (650, 2), (B, 4), (1, -1)):
        starts = list(base)
        starts[at] = v
        assert x.run(starts)[0] == 1, (at, v)


@pytest.mark.parametrize("which", [0, 1, 2])
@pytest.mark.parametrize("length", ["over", "far", "negative", "least"])
def test_append_lengths(cuda_lib, which, length):
    """A length beyond the table is flagged and all tokens of its sequence are left out, those whose own place lies inside it among
    them; sequence 1 has no new tokens, and its length is looked at all the same."""
    x = Appended([200, 300, 100], 40)
    cap = x.pool.max_pages * 64
    kv = [200, 300, 100]
    kv[which] = {"over": cap + 3, "far": (1 << 31) - 1, "negative": -1, "least": -(1 << 31)}[length]
    status, stored = x.run([0, 20, 20, 40], kv)
    assert status == 1
    assert stored == [which != 0] * 20 + [which != 2] * 20


# ------------------------------------------------------------------------------------------ the range of V
def spread(n, Hkv, dtype, level, jump, at):
    """Keys along one direction and queries along it: logits of `level`, and of `jump` more (log2) from row `at` on; the direction."""
    u = torch.zeros(D)
    u[:16] = 1.0                                            # 16 ones: products and their sums are exact in any order
    k = torch.zeros((Hkv, n, D))
    k[:, at:] = u * jump / 16
    return (k + u * level / 16).to(dtype).cuda(), u.to(dtype).cuda()


@pytest.mark.parametrize("form", ["prefill", "chunk", "decode", "prefix", "long prefix"])
@pytest.mark.parametrize("dtype,size", [(BF, 2.0 ** 100), (BF, 2.0 ** 115), (BF, 2.0 ** -100), (BF, 2.0 ** -125), (FP, 3e4), (FP, 2.0 ** -20)])
@pytest.mark.parametrize("jump", [7.0, 9.0, 36.0, 41.0])
def test_large_and_small_values(cuda_lib, form, dtype, size, jump):
    """Values of V whose sums fit into 32 bits, where the largest logit is far behind the first tile and above its maximum by just less
    or more than a reference is left to lag."""
    # (a long prefix of many heads is cut into chunks of several tiles: row 6100 lies inside one)
    n, Hq, Hkv, at = (12000, 8, 8, 6100) if form == "long prefix" else (700, 8, 2, 500)
    pool = Pool([n, 1], Hkv=Hkv, page=64, dtype=dtype, seed=6)
    k, u = spread(n, Hkv, dtype, 1.0, jump, at)
    pool.k_rows[0] = k
    pool.v_rows[0] = (torch.sign(pool.v_rows[0].float()) * size * torch.linspace(0.5, 1.0, D, device="cuda")).to(dtype)
    pool.k_rows[1], pool.v_rows[1] = k[:, :1], pool.v_rows[0][:, :1]
    for b in range(2):
        pool.write(b, 0, pool.k_rows[b], pool.v_rows[b])
    scale = math.log(2.0)                                   # logits in units of log2
    r = type("R", (), {})()
    if form in ("prefill", "chunk"):
        m = n if form == "prefill" else 3
        q = u.expand(m, Hq, D).contiguous()
        r = run_prefill(pool, q, [m], [n], Hq=Hq, scale=scale)
        check_prefill(pool, r, q, [m], [n], Hq=Hq, scale=scale)
        return
    q = u.expand(1, Hq, D).contiguous()
    p = cd.make_paged_params(B=1, Hq=Hq, Hkv=Hkv, page_size=64, n_pages=pool.n_pages, max_pages=pool.max_pages, dtype=dtype, softmax_scale=scale,
                             n_groups=1, max_prefix_pages=pool.max_pages)
    ws = workspace(p, 1)
    r.out, r.lse = torch.full_like(q, 7.0), torch.full((1, Hq), 7.0, device="cuda")
    if form == "decode":
        cd.calidrop_paged_decode(p, q, pool.K, pool.V, pool.table, i32([n]), r.out, r.lse, ws)
    else:
        cd.calidrop_paged_prefix_decode(p, q, pool.K, pool.V, i32([0, 1]), pool.table, i32([n]), pool.table[1:], i32([1]), r.out, r.lse, ws)
    assert status_of(ws) == 0
    if form == "decode":
        check_prefill(pool, r, q, [1], [n], Hq=Hq, scale=scale)
    else:
        own = type("P", (), dict(Hkv=Hkv, dtype=dtype, k_rows=pool.k_rows[1:], v_rows=pool.v_rows[1:]))
        check_prefill(own, r, q, [1], [1], Hq=Hq, scale=scale, prefix=[(pool, 0, n)])


# ------------------------------------------------------------------------------------------ a wait that runs out
WAIT = r'''
#include "paged_common.cuh"
using namespace calidrop;

// One CTA waits for a barrier at which nobody arrives, up to the limit of all waits, in a workspace whose word is `word`.
__global__ void wait_kernel(unsigned* word, int arrive) {
  __shared__ unsigned long long bar;
  __shared__ tc::Ctl ctl;
  if (threadIdx.x == 0) {
    ctl.abort = 0;
    ctl.status = word;
    tc::mbar_init(smem_u32(&bar), 1);
    tc::fence_mbar_init();
  }
  __syncthreads();
  if (threadIdx.x == 0 && arrive) tc::mbar_arrive(smem_u32(&bar));
  tc::mbar_wait(&ctl, smem_u32(&bar), 0, 0x100u);
  __syncthreads();
  paged_aborted(ctl);
}

extern "C" int run_wait(unsigned* word, int arrive) {
  wait_kernel<<<1, 32>>>(word, arrive);
  return (int)cudaDeviceSynchronize();
}
'''


def test_a_wait_that_runs_out_shows_beside_the_bits_of_bad_data(cuda_lib, tmp_path):
    """The waits of the prefill kernel, and how it reports them: a barrier that nobody arrives at, two seconds."""
    import ctypes
    import os
    import subprocess

    from paper_2507_19906_b200 import build

    src, lib = tmp_path / "wait.cu", tmp_path / "wait.so"
    src.write_text(WAIT)
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")] + build.NVCC_FLAGS + ["-I", build.CSRC, "-o", str(lib), str(src)])
    run = ctypes.CDLL(str(lib)).run_wait
    for word, arrive in ((0, 1), (2, 1), (0, 0), (3, 0)):
        w = i32([word])
        torch.cuda.synchronize()
        assert run(ctypes.c_void_p(w.data_ptr()), arrive) == 0
        got = w.item()
        if arrive:
            assert got == word
        else:
            assert got & 7 == word and got & ~7, hex(got)


# ------------------------------------------------------------------------------------------ more of the shared prefix
@pytest.mark.parametrize("what,bit", [("prefix page", 2), ("low prefix page", 2), ("page", 2), ("prefix length", 1), ("negative prefix length", 1),
                                      ("length", 1), ("negative length", 1)])
@pytest.mark.parametrize("members", [1, 20])
def test_bad_data_of_a_prefix_decode(cuda_lib, what, bit, members):
    """Flagged, and right for the sequences that it does not concern: the second group's, and in the first those whose own rows are not bad."""
    B = 2 * members
    x = Prefixed(B, [300, 260], 70)
    plens, kv = list(x.plens), list(x.kv)
    own = "prefix" not in what
    if what == "prefix page":
        x.prefix_table[0, 3] = x.pool.n_pages
    elif what == "low prefix page":
        x.prefix_table[0, 3] = -1
    elif what == "page":
        x.table[0, 0] = x.pool.n_pages + 5
    elif what.endswith("prefix length"):
        plens[0] = -3 if what.startswith("negative") else x.pool.max_pages * 32 + 1
        x.prefix_table[0].clamp_(min=0)             # a length is held to the table, and pages of it that exist are read
    else:
        kv[0] = -3 if what.startswith("negative") else x.pool.max_pages * 32 + 1
        x.table[0].clamp_(min=0)
    r = x.run([0, members, B], plens, kv)
    assert r.status == bit
    for b in range(1 if own else members, B):
        x.check(r, b, b // members)


def test_prefix_decode_repeats_itself(cuda_lib):
    """Bit for bit, in one workspace, whatever another call has left there."""
    x = Prefixed(60, [3000, 700, 64], 90, Hq=32, Hkv=8, page=64)
    first = x.run([0, 20, 59, 60])
    for b in (0, 19, 20, 58, 59):
        x.check(first, b, (b >= 20) + (b >= 59))
    for i in range(20):
        if i % 2:
            x.run([0, 1, 30, 31], kv=[1] * 60)
        r = x.run([0, 20, 59, 60])
        assert r.status == 0 and torch.equal(r.out, first.out) and torch.equal(r.lse, first.lse), i


@pytest.mark.parametrize("form", ["prefill", "decode", "prefix"])
@pytest.mark.parametrize("dtype", [BF, FP])
def test_a_key_at_minus_infinity_drops_out(cuda_lib, form, dtype):
    """Logits of -inf weigh nothing, in the first tile, inside one and at the end; a token that sees no others gets zeros."""
    n, Hq, Hkv = 300, 8, 2
    G = Hq // Hkv
    pool = Pool([n, 1], Hkv=Hkv, page=64, dtype=dtype, seed=1)
    gone = torch.zeros(n, dtype=torch.bool, device="cuda")
    gone[[0, 1, 129, 200, n - 1]] = True
    finite = pool.k_rows[0].clone()
    pool.k_rows[0][:, gone, 0] = -math.inf
    pool.write(0, 0, pool.k_rows[0], pool.v_rows[0])
    finite[:, gone] = 0
    T = n if form == "prefill" else 1
    q = queries(T, Hq, dtype, 2)
    q[..., 0] = q[..., 0].abs() + 0.5
    p = cd.make_paged_params(B=1, Hq=Hq, Hkv=Hkv, page_size=64, n_pages=pool.n_pages, max_pages=pool.max_pages, dtype=dtype, n_groups=1,
                             max_prefix_pages=pool.max_pages)
    ws, out, lse = workspace(p, T), torch.full_like(q, 7.0), torch.full((T, Hq), 7.0, device="cuda")
    if form == "prefill":
        cd.calidrop_paged_prefill(p, q, pool.K, pool.V, pool.table, i32([0, n]), i32([n]), out, lse, ws)
    elif form == "decode":
        cd.calidrop_paged_decode(p, q, pool.K, pool.V, pool.table, i32([n]), out, lse, ws)
    else:
        cd.calidrop_paged_prefix_decode(p, q, pool.K, pool.V, i32([0, 1]), pool.table, i32([n]), pool.table[1:], i32([0]), out, lse, ws)
    assert status_of(ws) == 0
    t = torch.arange(n, device="cuda")
    seen = (t <= (t if form == "prefill" else t[-1:])[:, None]) & ~gone
    for hq in range(Hq):
        ref = attention64(q[:, hq], finite[hq // G], pool.v_rows[0][hq // G], seen, 1 / math.sqrt(D))
        check_rows(out[:, hq], lse[:, hq], ref, dtype, n, f"head {hq}")


# ------------------------------------------------------------------------------------------ long appends
@pytest.mark.parametrize("dtype,Hq,Hkv,T,rot,interleaved,page", [
    (BF, 32, 8, 592, 128, False, 64),            # the most tokens of which a lane takes one row
    (BF, 32, 8, 593, 128, False, 64),            # and the fewest of which it takes four
    (BF, 28, 4, 901, 64, True, 16),
    (FP, 5, 1, 5001, 96, False, 128),            # seven rows a token: most lanes have fewer than four
    (FP, 16, 16, 700, 128, True, 256),
])
@pytest.mark.parametrize("with_q", [True, False])
def test_long_appends(cuda_lib, dtype, Hq, Hkv, T, rot, interleaved, page, with_q):
    """Both forms of the kernel, against the definition."""
    if not with_q:
        T = T * (Hq + 2 * Hkv) // (2 * Hkv)                  # as many rows
    lens = [T // 3, 0, T - T // 3 - 1, 1]
    old = [7, 30, 0, 70]
    kv = [a + b for a, b in zip(lens, old)]
    pool = Pool(kv, Hkv=Hkv, page=page, dtype=dtype, seed=2)
    g = torch.Generator().manual_seed(4)
    q, k, v = (torch.randn((T, h, D), generator=g).to(dtype).cuda() for h in (Hq, Hkv, Hkv))
    cs = table_of_angles(max(kv), rot)
    p = cd.make_paged_params(B=4, Hq=Hq, Hkv=Hkv, page_size=page, n_pages=pool.n_pages, max_pages=pool.max_pages, dtype=dtype, rot_dim=rot,
                             interleaved=interleaved, max_pos=max(kv))
    ws, q_out = workspace(p, T), torch.full((T, Hq, D), 7.0, dtype=dtype, device="cuda")
    cd.calidrop_paged_append(p, q if with_q else None, k, v, None, cs, pool.K, pool.V, pool.table, starts(lens), i32(kv), q_out, ws)
    assert status_of(ws) == 0
    place = torch.cat([torch.arange(o, o + n) for o, n in zip(old, lens)]).cuda()
    got_k, got_v = (torch.cat([pool.read(x, b, kv[b])[:, old[b]:].transpose(0, 1) for b in range(4)]) for x in (pool.K, pool.V))
    assert torch.equal(got_v, v)
    for got, x in [(got_k, k)] + ([(q_out, q)] if with_q else []):
        ref, size = turned64(x, cs[place], rot, interleaved)
        # two products and a sum in 32 bits (each half a step of 2^-23), then the rounding
        assert ((got.double() - ref).abs() <= HALF[dtype] * ref.abs() + 3 * 2.0 ** -24 * size + SMALL[dtype]).all()
        assert torch.equal(got[..., rot:], x[..., rot:])
    for b in range(4):                                        # the rows ahead are as they were
        assert torch.equal(pool.read(pool.K, b, old[b]), pool.k_rows[b][:, :old[b]])
        assert torch.equal(pool.read(pool.V, b, old[b]), pool.v_rows[b][:, :old[b]])
    if not with_q:
        assert (q_out == 7.0).all()
