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


def shorter(t, s, dim):
    return torch.zeros(tuple(n - (d == dim) for d, n in enumerate(s)), dtype=BF if t == "half" else t)


# (the tokens of append and prefill are counted by k and q)
@pytest.mark.parametrize("entry,name", [c for c in CASES if c not in (("append", "k"), ("prefill", "q"))])
def test_too_few_rows(entry, name):
    kind, shape = next((t, s) for n, t, s in ENTRIES[entry] if n == name)
    with pytest.raises(ValueError, match=f"{name} is too small"):
        call(entry, arguments(entry, **{name: shorter(kind, shape, 0)}))
    with pytest.raises(ValueError, match=f"{name} is too small"):
        call(entry, arguments(entry, **{name: shorter(kind, shape, 0).flatten()}))
    # more rows are no fault, and where all is packed their dimensions neither
    more = torch.zeros((shape[0] + 3, *shape[1:]), dtype=BF if kind == "half" else kind)
    for x in (more, more.flatten()):
        with pytest.raises(ValueError, match="CUDA device"):
            call(entry, arguments(entry, **{name: x}))


@pytest.mark.parametrize("entry,name", [c for c in CASES if c[1] not in ("positions", "q_start", "kv_len", "group_start", "prefix_len")])
def test_rows_of_another_length(entry, name):
    kind, shape = next((t, s) for n, t, s in ENTRIES[entry] if n == name)
    with pytest.raises(ValueError, match=f"^{name}"):
        call(entry, arguments(entry, **{name: shorter(kind, shape, 1)}))


@pytest.mark.parametrize("entry", ENTRIES)
def test_tables_and_pages_in_another_layout(entry):
    wide = torch.zeros((B, MAX_PAGES + 1), dtype=I32)
    with pytest.raises(ValueError, match="^block_table"):
        call(entry, arguments(entry, block_table=wide))
    swapped = torch.zeros((N_PAGES, PAGE, HKV, D), dtype=BF)
    for name in ("K_pages", "V_pages"):
        with pytest.raises(ValueError, match=f"^{name}"):
            call(entry, arguments(entry, **{name: swapped}))
    # of a single sequence's table the rest is not looked at
    one = dict(block_table=torch.zeros((1, MAX_PAGES + 1), dtype=I32), group_start=torch.zeros(2, dtype=I32))
    with pytest.raises(ValueError, match="CUDA device"):
        call(entry, arguments(entry, **{k: v for k, v in one.items() if k in [n for n, *_ in ENTRIES[entry]]}), B=1)


def test_strided_queries_and_halves_of_a_pool():
    """The views that the parameters' strides describe, and those that they do not."""
    x = torch.zeros((T, HQ + 2 * HKV, D), dtype=BF)
    q, k, v = x[:, :HQ], x[:, HQ:HQ + HKV], x[:, HQ + HKV:]
    both = torch.zeros((N_PAGES, 2, HKV, PAGE, D), dtype=BF)
    strides = dict(q_stride=q.stride(0), k_stride=k.stride(0), v_stride=v.stride(0), page_stride=both.stride(0))
    args = arguments("append", q=q, k=k, v=v, K_pages=both[:, 0], V_pages=both[:, 1])
    with pytest.raises(ValueError, match="CUDA device"):
        call("append", args, **strides)
    with pytest.raises(ValueError, match="^q is too small"):          # fewer tokens than keys
        call("append", [q[:-1]] + args[1:], **strides)
    with pytest.raises(ValueError, match="^q is too small"):          # a flat tensor has no stride between its tokens
        call("append", [torch.zeros(x.numel(), dtype=BF)] + args[1:], **strides)
    with pytest.raises(ValueError, match="CUDA device"):              # no queries: what stands for their output is not looked at
        call("append", [None] + args[1:9] + [args[9], torch.zeros(1, dtype=BF), args[11]], **strides)
