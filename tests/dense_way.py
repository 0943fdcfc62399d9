"""The two ways of the dense operators' binding, as a fixture."""
import pytest
import torch

from paper_2110_09132_amd import dense


@pytest.fixture(params=["short", "long"])
def way(request):
    """The binding with its short way in C, and without (every call then goes the long way)."""
    api = getattr(torch.Tensor, "__dlpack_c_exchange_api__", None)
    assert dense._native.use(api if request.param == "short" else None, torch.Tensor,
                             torch.nn.Parameter) == (request.param == "short")
    yield request.param
    dense._native.use(api, torch.Tensor, torch.nn.Parameter)
