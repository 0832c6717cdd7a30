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
