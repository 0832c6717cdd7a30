"""What the entry points over a cache in pages refuse: checked on the host, ahead of every CUDA call, so no device is needed."""
import ctypes

import pytest
import torch

from paper_2507_19906_b200 import binding as cd
from paper_2507_19906_b200 import build as cdbuild

GOOD = dict(B=3, Hq=8, Hkv=2, page_size=64, n_pages=20, max_pages=5)


@pytest.fixture(scope="module")
def lib():
    cdbuild.build()
    return cd.load()


@pytest.fixture(scope="module")
def at():
    """An aligned host address: never dereferenced."""
    buf = (ctypes.c_char * 4096)()
    yield (ctypes.addressof(buf) + 255) & ~255
    del buf


def calls(names, lib, p, a, n=4, size=1 << 40, **other):
    """The entry points `names`, each with good arguments but for `other`, which it has to refuse: {name: status}.  (No others:
    on a machine with a device they would run on these addresses.)"""
    v = dict.fromkeys(("q", "k", "v", "positions", "cos_sin", "K", "V", "table", "q_start", "kv_len", "out", "lse", "ws", "groups",
                       "prefix_table", "prefix_len"), a)
    v.update(other)
    g = {k: ctypes.c_void_p(x) for k, x in v.items()}
    pp = ctypes.byref(p)
    run = {
        "append": lambda: lib.calidrop_paged_append(pp, n, g["q"], g["k"], g["v"], g["positions"], g["cos_sin"], g["K"], g["V"],
                                                    g["table"], g["q_start"], g["kv_len"], g["out"], g["ws"], size, None),
        "prefill": lambda: lib.calidrop_paged_prefill(pp, n, g["q"], g["K"], g["V"], g["table"], g["q_start"], g["kv_len"], g["out"],
                                                      g["lse"], g["ws"], size, None),
        "decode": lambda: lib.calidrop_paged_decode(pp, g["q"], g["K"], g["V"], g["table"], g["kv_len"], g["out"], g["lse"], g["ws"],
                                                    size, None),
        "prefix": lambda: lib.calidrop_paged_prefix_decode(pp, g["q"], g["K"], g["V"], g["groups"], g["prefix_table"], g["prefix_len"],
                                                           g["table"], g["kv_len"], g["out"], g["lse"], g["ws"], size, None),
    }
    return {name: run[name]() for name in names}


ALL = {"append", "prefill", "decode", "prefix"}

BAD_PARAMS = [
    (dict(B=0), cd.INVALID_ARG), (dict(Hq=7), cd.INVALID_ARG), (dict(Hkv=0), cd.INVALID_ARG), (dict(D=64), cd.UNSUPPORTED),
    (dict(Hq=18, Hkv=2), cd.UNSUPPORTED), (dict(B=4097), cd.UNSUPPORTED), (dict(dtype=2), cd.UNSUPPORTED),
    (dict(page_size=8), cd.UNSUPPORTED), (dict(page_size=48), cd.UNSUPPORTED), (dict(page_size=512), cd.UNSUPPORTED),
    (dict(n_pages=0), cd.INVALID_ARG), (dict(max_pages=0), cd.INVALID_ARG), (dict(max_pages=1 << 25), cd.INVALID_ARG),
    (dict(window=-1), cd.INVALID_ARG), (dict(n_sink=-1), cd.INVALID_ARG), (dict(softmax_scale=-1.0), cd.INVALID_ARG),
    (dict(softmax_scale=float("nan")), cd.INVALID_ARG), (dict(rot_dim=24, max_pos=9), cd.UNSUPPORTED),
    (dict(rot_dim=144, max_pos=9), cd.UNSUPPORTED), (dict(rot_dim=128, max_pos=0), cd.INVALID_ARG),
    (dict(n_groups=4, max_prefix_pages=1), cd.INVALID_ARG), (dict(n_groups=1, max_prefix_pages=0), cd.INVALID_ARG),
    (dict(q_stride=8 * 128 - 8), cd.INVALID_ARG), (dict(q_stride=8 * 128 + 4), cd.INVALID_ARG), (dict(k_stride=128), cd.INVALID_ARG),
    (dict(v_stride=-256), cd.INVALID_ARG), (dict(page_stride=2 * 64 * 128 - 128), cd.INVALID_ARG),
]


@pytest.mark.parametrize("bad,status", BAD_PARAMS)
def test_parameters(lib, at, bad, status):
    p = cd.make_paged_params(**{**GOOD, "n_groups": 1, "max_prefix_pages": 2, **bad})
    assert cd.calidrop_paged_workspace_bytes(p, 4) == 0
    assert set(calls(ALL, lib, p, at).values()) == {status}


def test_arguments(lib, at):
    p = cd.make_paged_params(**GOOD, rot_dim=128, max_pos=10, n_groups=1, max_prefix_pages=2)
    need = cd.calidrop_paged_workspace_bytes(p, 4)
    assert need % 256 == 0 and need > 0
    def refused(names, status=cd.INVALID_ARG, **other):
        got = calls(names, lib, p, at, **other)
        assert set(got.values()) == {status}, (got, other)

    for name in ("K", "V", "table", "kv_len", "ws"):
        refused(ALL, **{name: None})
    for name in ("K", "V", "out"):
        refused(ALL, **{name: at + 8})
    refused({"prefill", "decode", "prefix"}, q=None)
    refused(ALL, q=at + 2)
    refused({"prefill", "decode", "prefix"}, lse=at + 2)
    refused({"append", "prefill"}, q_start=None)
    refused({"append"}, k=None)
    refused({"append"}, v=at + 8)
    refused({"append"}, cos_sin=None)
    refused({"append"}, positions=at + 1)
    refused({"prefix"}, groups=None)
    refused({"prefix"}, prefix_table=None)
    refused({"prefix"}, prefix_len=at + 2)
    refused(ALL, ws=at + 16)
    refused({"append", "prefill"}, n=-1)
    refused({"append", "prefill"}, n=(1 << 25) + 1)
    refused({"append", "prefill"}, cd.WORKSPACE_TOO_SMALL, size=need - 256)
    # in place over strided queries: the packed output would overlap them
    p.q_stride = 16 * 128
    refused({"append"})
    p.q_stride = 0
    # no window over a shared prefix, and no prefix without groups
    p.window = 5
    refused({"prefix"}, cd.UNSUPPORTED)
    p.window, p.n_groups = 0, 0
    refused({"prefix"})


def test_sizes_grow_with_the_tokens(lib):
    p = cd.make_paged_params(**GOOD)
    sizes = [cd.calidrop_paged_workspace_bytes(p, n) for n in (0, 1, 3, 100, 5000, 1 << 20)]
    assert sizes == sorted(sizes) and sizes[0] > 0
    assert cd.calidrop_paged_workspace_bytes(p, -1) == 0


def test_binding_takes_structures_and_tensors_for_what_they_are(lib):
    p = cd.make_paged_params(**GOOD)
    none = [None] * 8
    for bad in (None, 0, b"", bytes(p), cd.Params(), ctypes.byref(p)):
        with pytest.raises(TypeError):
            cd.calidrop_paged_decode(bad, *none)
    for host in (torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(4)):
        with pytest.raises((ValueError, RuntimeError)):
            cd.calidrop_paged_decode(p, host, *none[1:])
        with pytest.raises((ValueError, RuntimeError)):
            cd.calidrop_paged_prefill(p, host, *none)
    with pytest.raises((TypeError, AttributeError)):
        cd.calidrop_paged_append(p, *[None] * 12)          # no tensor to count the tokens of
    assert ctypes.sizeof(cd.PagedParams) == 16 * 4 + 4 * 8
