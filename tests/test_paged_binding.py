"""What the binding of the entry points over a cache in pages refuses, ahead of the library: no device is needed."""
import pytest
import torch

from paper_2507_19906_b200 import binding as cd
from paper_2507_19906_b200 import build as cdbuild

B, HQ, HKV, PAGE, N_PAGES, MAX_PAGES, D = 3, 8, 2, 64, 20, 5, 128
BF, I32, F32 = torch.bfloat16, torch.int32, torch.float32


@pytest.fixture(scope="module", autouse=True)
def lib():
    cdbuild.build()
    return cd.load()


def params(**other):
    return cd.make_paged_params(**{**dict(B=B, Hq=HQ, Hkv=HKV, page_size=PAGE, n_pages=N_PAGES, max_pages=MAX_PAGES), **other})


class Sub(torch.Tensor):
    pass


def test_tensors_of_a_subclass_have_a_device_too():
    """The address of a tensor on the host is refused whatever its class."""
    x = torch.zeros((B, HQ, D), dtype=BF)
    for q in (x, x.as_subclass(Sub), torch.nn.Parameter(x)):
        with pytest.raises(ValueError, match="CUDA device"):
            cd.calidrop_paged_decode(params(), q, *[None] * 7)
        with pytest.raises(ValueError, match="CUDA device"):
            cd.calidrop_paged_prefill(params(), q, *[None] * 8)


# The arguments of each entry point behind the parameters: name, element type ("half": that of the parameters), and shape.
T = 4
ROWS = lambda n, h: (n, h, D)
TABLES = [("block_table", I32, (B, MAX_PAGES)), ("q_start", I32, (B + 1,)), ("kv_len", I32, (B,))]
PAGES = [("K_pages", "half", (N_PAGES, HKV, PAGE, D)), ("V_pages", "half", (N_PAGES, HKV, PAGE, D))]
WS = ("workspace", torch.uint8, (0,))
ENTRIES = {
    "append": [("q", "half", ROWS(T, HQ)), ("k", "half", ROWS(T, HKV)), ("v", "half", ROWS(T, HKV)), ("positions", I32, (T,)),
               ("cos_sin", F32, (10, D))] + PAGES + TABLES + [("q_out", "half", ROWS(T, HQ)), WS],
    "prefill": [("q", "half", ROWS(T, HQ))] + PAGES + TABLES + [("out", "half", ROWS(T, HQ)), ("lse", F32, (T, HQ)), WS],
    "decode": [("q", "half", ROWS(B, HQ))] + PAGES + [TABLES[0], TABLES[2], ("out", "half", ROWS(B, HQ)), ("lse", F32, (B, HQ)), WS],
    "prefix_decode": [("q", "half", ROWS(B, HQ))] + PAGES + [("group_start", I32, (2,)), ("prefix_table", I32, (1, 7)), ("prefix_len", I32, (1,)),
                                                             TABLES[0], TABLES[2], ("out", "half", ROWS(B, HQ)), ("lse", F32, (B, HQ)), WS],
}


def arguments(entry, half=BF, **other):
    """Host tensors that are right but for their device (which is looked at last), with `other` in place of some."""
    return [other[n] if n in other else torch.zeros(s, dtype=half if t == "half" else t) for n, t, s in ENTRIES[entry]]


def call(entry, args, **p):
    p = params(**{**dict(rot_dim=128, max_pos=10, n_groups=1, max_prefix_pages=7), **p})
    return getattr(cd, "calidrop_paged_" + entry)(p, *args)


CASES = [(e, n) for e, rows in ENTRIES.items() for n, *_ in rows if n != "workspace"]


@pytest.mark.parametrize("entry", ENTRIES)
@pytest.mark.parametrize("half", [BF, torch.float16])
def test_right_tensors_lack_nothing_but_the_device(entry, half):
    with pytest.raises(ValueError, match="CUDA device"):
        call(entry, arguments(entry, half), dtype=half)
    # parameters that the library refuses are its own to name: no tensor is measured by them
    with pytest.raises(ValueError, match="CUDA device"):
        call(entry, arguments(entry, half), dtype=half, page_size=48)


@pytest.mark.parametrize("entry,name", CASES)
def test_element_types(entry, name):
    kind, shape = next((t, s) for n, t, s in ENTRIES[entry] if n == name)
    for wrong in (torch.int64, I32, F32, BF, torch.float16, torch.int16, torch.float64):
        if wrong is (BF if kind == "half" else kind):
            continue
        for x in (torch.zeros(shape, dtype=wrong), torch.zeros(shape, dtype=wrong).as_subclass(Sub)):
            with pytest.raises(ValueError, match=f"{name} has elements of type"):
                call(entry, arguments(entry, **{name: x}))
    if kind == "half":                               # a bf16 tensor among fp16 parameters
        x = torch.zeros(shape, dtype=BF)
        with pytest.raises(ValueError, match=f"{name} has elements of type BFloat16, Half expected"):
            call(entry, arguments(entry, torch.float16, **{name: x}), dtype=torch.float16)
