"""Sums of dweight and dbias over very many rows: their rounding errors grow as
those of sums in two levels, not with the rows that a lane takes.

Equal rows x and dy = 1, so that dweight is n xh and dbias n exactly (n < 2^24),
and every rounding of a running sum that favours one side adds up.  Bound: a
float32 sum of t terms is off by at most t u of their magnitudes (u = 2^-24).  A
lane adds 32 rows at a time and then those sums, a block up to 32 lanes of a
column, and the 512 blocks are added 32 at a time: with rows = n / 512, as if one
lane took all rows of its block, 32 + rows / 32 + 32 + 32 + 16 terms in a row.
xh is formed from the mean and rstd that are given with two roundings.
"""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
u = 2.0 ** -24


@pytest.mark.parametrize("n,d,dtype", [
    (16_000_000, 16, torch.float32), (2_000_000, 250, torch.float32), (1_000_000, 1024, torch.float32),
    (500_000, 4096, torch.float32), (2_000_000, 2048, torch.bfloat16), (500_000, 4096, torch.float16),
    (400_000, 8192, torch.bfloat16), (400_000, 16_384, torch.float16), (400_000, 8190, torch.bfloat16),
    (400_000, 3001, torch.bfloat16), (400_000, 8196, torch.bfloat16), (400_000, 16_392, torch.float16)])
def test_many_equal_rows(n, d, dtype):
    print("case", n, d, dtype, flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(d)
    row = torch.randn(d, generator=g, device=DEV).to(dtype)
    X = row.repeat(n, 1)
    mean = torch.full((n,), float(row.double().mean()), dtype=torch.float32, device=DEV)
    rstd = torch.full((n,), float(1 / row.double().std(correction=0)), dtype=torch.float32, device=DEV)
    dX, dg, db = km.layernorm_backward(torch.ones_like(X), X, mean, rstd)
    del dX, X
    xh = (row.double() - mean[0].double()) * rstd[0].double()
    terms = 32 + n / 512 / 32 + 32 + 32 + 16
    off = ((dg.double() / n - xh).abs() / (u * xh.abs())).max()
    assert off <= terms + 2, (float(off), terms)
    assert ((db.double() - n).abs() <= terms * u * n).all()
    torch.cuda.empty_cache()
