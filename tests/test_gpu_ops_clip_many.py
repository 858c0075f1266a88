"""Norm and scaling over thousands of tensors: more than a launch takes by far, and more
sums than blocks of the second pass."""
import pytest
import torch

from test_gpu_ops_clip import DEV, TYPES, _check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("count", [1000, 5000])
def test_thousands_of_tensors(count):
    g = torch.Generator(device=DEV)
    g.manual_seed(count)
    ts = [torch.randn(1 + (i * 37) % 311, generator=g, device=DEV).to(TYPES[i % 3]) for i in range(count)]
    ts[count // 2] = torch.randn(100_003, generator=g, device=DEV)
    for share in (0.3, 2.0):
        _check(ts, share)
