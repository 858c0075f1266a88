"""Products in 8 bits at the ends of the exponents' range: values that their power of
two takes out of a smaller type's range, or of float32's, while the product is in it.

A product of two e4m3 values has 8 bits and is the only one of its sum here, so every
result is that product, rounded once to the result's type."""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
F64 = torch.float64


def _blocks(values, byte):
    e = torch.full(values.shape[:-1] + ((values.shape[-1] + 127) // 128,), byte, dtype=torch.uint8, device=DEV)
    return km.BlockRows(values.to(torch.float8_e4m3fn), e)


def _rows(n, din, at, v, byte):
    x = torch.zeros(n, din, device=DEV)
    x[:, at] = v
    return _blocks(x, byte)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,din", [(3, 128), (40, 200), (100, 256), (100, 77), (5000, 256)])
def test_products_of_far_exponents(n, din, dtype):
    """Rows down to 2^-136 and up to 1.75 2^135, the weight's power the opposite."""
    plan = km.cluster_sort(torch.zeros(n, dtype=torch.int32, device=DEV), 1)
    at = din - 1
    for byte, other in ((0, 254), (1, 250), (3, 247), (9, 240), (238, 20), (247, 10), (250, 4), (254, 0)):
        for v in (2.0 ** -9, 3 * 2.0 ** -9, 2.0 ** -6, 1.875 * 2.0 ** -6, 1.0, 1.75 * 2.0 ** 8):
            X = _rows(n, din, at, v, byte)
            w = _rows(65, din, at, 1.25, other)
            W = km.BlockRows(w.values[None], w.exponents[None])
            want = torch.tensor(1.25 * v * 2.0 ** (byte + other - 254), dtype=F64).to(dtype)
            got = km.cluster_linear_fp8(X, W, plan, dtype=dtype)
            assert bool((got == want.to(DEV)).all()), (byte, other, v, float(got[0, 0]), float(want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 100, 5000])
def test_rows_of_the_least_and_largest_float32(n, dtype):
    """Quantised rows: float32's largest value stands for 2^128, its subnormals for themselves."""
    plan = km.cluster_sort(torch.zeros(n, dtype=torch.int32, device=DEV), 1)
    for v, stands, power in ((torch.finfo(torch.float32).max, 2.0 ** 128, -120), (2.0 ** -133, 2.0 ** -133, 120),
                             (5 * 2.0 ** -135, 5 * 2.0 ** -135, 120)):
        X = torch.zeros(n, 130, device=DEV)
        X[:, 3] = v
        W = km.quantize_blocks(torch.full((1, 64, 130), 2.0 ** power, device=DEV))
        want = torch.tensor(stands * 2.0 ** power, dtype=F64).to(dtype).to(DEV)
        assert bool((km.cluster_linear_fp8(X, W, plan, dtype=dtype) == want).all()), v


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [3, 100, 5000])
def test_a_byte_of_255_is_nan_whatever_the_value(n, dtype):
    plan = km.cluster_sort(torch.zeros(n, dtype=torch.int32, device=DEV), 1)
    for v in (0.0, 1.0):
        q, W = _blocks(torch.full((n, 256), v, device=DEV), 127), _blocks(torch.ones(1, 64, 256, device=DEV), 127)
        q.exponents[n - 1, 1] = 255
        got = km.cluster_linear_fp8(q, W, plan, dtype=dtype)
        assert bool(got[n - 1].isnan().all()) and bool((got[:n - 1] == 256 * v).all())
        q.exponents.fill_(127)
        W.exponents[0, 5, 0] = 255
        got = km.cluster_linear_fp8(q, W, plan, dtype=dtype)
        assert bool(got[:, 5].isnan().all()) and bool((got[:, :5] == 256 * v).all())
