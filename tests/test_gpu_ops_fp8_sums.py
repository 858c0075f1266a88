"""Sums of 8-bit products of very uneven size: one large product among each eight
consecutive ones, of one sign or of signs that cancel, against float64.

Tolerances.  Products of two e4m3 values are exact in float32 and the scales powers of
two.  Float32 results: a float32 sum of t products, in any order, is off by at most 2 t u
times the sum of the magnitudes (u = 2^-24), and the result is the sum.  Results of 16
bits: of eight consecutive products each loses less than 2^-13 2^m, m being the largest
sum of two exponents among them, so the eight lose at most 2^-10 2^m, beside the float32
sum and one rounding of the result (half a step, U)."""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
u = 2.0 ** -24
F64 = torch.float64


def _case(n, din, dout, cancel):
    """Every eighth product is 2^9 or more (with alternate signs where they cancel), the
    others are up to 2^-4: what lies 13 bits and more below the large ones."""
    g = torch.Generator(device=DEV)
    g.manual_seed(n + din)
    rand = lambda *s: torch.rand(*s, generator=g, device=DEV)
    at = torch.arange(din, device=DEV)
    big = at % 8 == (at // 8 * 5 + 3) % 8
    sign = torch.where(at // 8 % 2 == 1, -1.0, 1.0) if cancel else torch.ones(din, device=DEV)
    x = torch.where(big, 32.0 * sign, 0.125 + 0.125 * rand(n, din)).to(torch.float8_e4m3fn)
    w = torch.where(big, 16.0, 0.125 + 0.125 * rand(1, dout, din)).to(torch.float8_e4m3fn)
    blocks = (din + 127) // 128
    byte = lambda *s: torch.randint(120, 134, s, generator=g, device=DEV).to(torch.uint8)
    return km.BlockRows(x, byte(n, 1).expand(n, blocks).contiguous()), \
        km.BlockRows(w, byte(1, dout, 1).expand(1, dout, blocks).contiguous()), 9


@pytest.mark.parametrize("cancel", [False, True])
@pytest.mark.parametrize("n,din,dout", [(5, 64, 80), (40, 1024, 48), (100, 128, 200), (100, 77, 65), (5000, 128, 512),
                                        (5000, 1024, 2304)])
def test_one_large_product_of_eight(n, din, dout, cancel):
    X, W, m = _case(n, din, dout, cancel)
    plan = km.cluster_sort(torch.zeros(n, dtype=torch.int32, device=DEV), 1)
    two = lambda e: torch.exp2(e.double() - 127)
    scale = two(X.exponents[:, :1]) * two(W.exponents[0, :, 0])[None]
    x, w = X.values.float().to(F64), W.values[0].float().to(F64)
    want, most = (x @ w.T) * scale, (x.abs() @ w.abs().T) * scale
    sums = 2 * din * u * most
    y = km.cluster_linear_fp8(X, W, plan, dtype=torch.float32).to(F64)
    assert bool(((y - want).abs() <= sums).all())
    lost = (din + 7) // 8 * 2.0 ** (m - 10) * scale
    for dtype in (torch.bfloat16, torch.float16):
        got = km.cluster_linear_fp8(X, W, plan, dtype=dtype).to(F64)
        tol = sums + lost
        tol = tol + U[dtype] * (want.abs() + tol) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
        near = (got - want).abs() <= tol
        if dtype == torch.float16:   # beyond its range: infinity
            near |= ((want.abs() + tol) >= torch.finfo(dtype).max) & got.isinf()
        assert bool(near.all()), dtype
        # Float32 results rounded afterwards keep float32 sums.
        back = y.to(torch.float32).to(dtype).to(F64)
        tol = sums + U[dtype] * (want.abs() + sums) + (2.0 ** -25 if dtype == torch.float16 else 0.0)
        near = (back - want).abs() <= tol
        if dtype == torch.float16:
            near |= ((want.abs() + tol) >= torch.finfo(dtype).max) & back.isinf()
        assert bool(near.all()), dtype
