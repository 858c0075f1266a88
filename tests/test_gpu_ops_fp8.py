"""Rows in 8 bits (quantize_blocks, dequantize_blocks) against the definition in
float64, bit for bit, and their products with one weight per cluster
(cluster_linear_fp8) against float64 products of the values that they stand for.

Tolerance of a product.  Products of two e4m3 values are exact in float32, the
scales are powers of two, and a float32 sum of t of them, in any order, is off
by at most 2 t u times the sum of the magnitudes (u = 2^-24; the factor 2
covers sums inside a matrix instruction that are not rounded to nearest).  The
result is rounded once to its type (U).

Results of 16 bits come from the 8-bit matrix instructions, which align each 8
consecutive products to the one of the largest exponent and drop what lies more
than 13 bits below it: each product loses less than 2^-13 times 2^m, m being the
largest sum of two exponents among the 8 (of a subnormal value -6), so 8 of
them at most 2^-10 2^m.  Float32 results come from bfloat16 instructions, which
do not.
"""
import pytest
import torch

import paper_1902_09527_amd as km

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
U = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
u = 2.0 ** -24
TYPES = [torch.float32, torch.bfloat16, torch.float16]
F64 = torch.float64


def _two(power):
    return ((power.long() + 1023) << 52).view(F64)


def _defined(x):
    """(values, exponent bytes) of rows on the CPU, in float64."""
    x, d = x.cpu().to(F64), x.shape[-1]
    values, bytes_ = torch.empty_like(x), []
    for at in range(0, d, 128):
        part = x[..., at:at + 128]
        most = torch.where(part.isfinite(), part.abs(), 0.0).amax(-1, keepdim=True)
        frac, power = torch.frexp(most / 448.0)   # exact next to powers of two: most has at most 24 bits
        power = torch.where(most > 0, torch.where(frac > 0.5, power, power - 1), -126).clamp_min(-126)
        v = part * _two(-power)
        _, top = torch.frexp(torch.where(v.isfinite(), v, 0.0))
        step = _two((top - 1).clamp_min(-6) - 3)
        v = torch.where(v.isfinite(), torch.round(v / step) * step, float("nan"))
        values[..., at:at + 128] = v
        bytes_.append(power + 127)
    return values, torch.cat(bytes_, -1).to(torch.uint8)


def _stands(q):
    p = (q.exponents.int() - 127).repeat_interleave(128, -1)[..., :q.shape[-1]]
    return q.values.to(torch.float32).to(F64) * _two(p)


def _quantized(x):
    q = km.quantize_blocks(x)
    values, bytes_ = _defined(x)
    assert q.values.dtype == torch.float8_e4m3fn and torch.equal(q.exponents.cpu(), bytes_)
    got = q.values.cpu().float().to(F64)
    assert torch.equal(got.isnan(), values.isnan())
    assert torch.equal(got.nan_to_num(0.0), values.nan_to_num(0.0))
    return q


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n,d", [(1, 1), (3, 7), (5, 8), (2, 127), (2, 128), (7, 129), (33, 250), (1000, 256),
                                 (130, 1000), (4, 4100), (2, 16_385), (20_000, 40), (0, 64)])
def test_quantize(n, d, dtype):
    print("case", n, d, dtype, flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(n + d)
    x = torch.randn(n, d, generator=g, device=DEV) * torch.exp(2 * torch.randn(d, generator=g, device=DEV))
    q = _quantized(x.to(dtype))
    for t in TYPES:
        back = km.dequantize_blocks(q, t)
        assert back.dtype == t and torch.equal(back, _stands(q).to(t))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_special_values(dtype):
    """Zeros, values between two e4m3 values and at the border of two exponents,
    the type's least and largest values, infinities and NaN."""
    top, tiny = torch.finfo(dtype).max, torch.finfo(dtype).smallest_normal
    x = torch.zeros(12, 256, device=DEV)
    x[1, 0], x[1, 1] = 448, -0.0
    x[2, 0] = 448 * (1 + torch.finfo(dtype).eps)
    x[3] = torch.linspace(-448, 448, 256)
    x[4, :128] = torch.arange(128) * 2.0 ** -10          # subnormal results and their ties
    x[4, 127] = 448
    x[5] = float("inf")
    x[6, :5] = torch.tensor([float("nan"), float("inf"), float("-inf"), 3.0, -5.0])
    x[7] = top
    x[8, :3] = torch.tensor([top, 1.0, tiny])
    x[9] = tiny
    x[9, 5] = tiny * torch.finfo(dtype).eps              # the type's least value
    x[10, 130] = tiny * torch.finfo(dtype).eps * 3
    x[11] = 448.0 * 2.0 ** -12
    _quantized(x.to(dtype))


@pytest.mark.parametrize("dtype", TYPES)
def test_quantize_strided_and_weights(dtype):
    x = torch.randn(50, 203, device=DEV).to(dtype)
    for view in (x[:, :200], x[:, 1:194], x[::2, 3:131]):
        _quantized(view)
    w = torch.randn(5, 33, 130, device=DEV).to(dtype)
    q, flat = km.quantize_blocks(w), km.quantize_blocks(w.view(165, 130))
    assert q.shape == w.shape and q.exponents.shape == (5, 33, 2)
    assert torch.equal(q.values.view(165, 130).view(torch.uint8), flat.values.view(torch.uint8))
    assert torch.equal(q.exponents.view(165, 2), flat.exponents)
    assert torch.equal(km.dequantize_blocks(q).view(165, 130), km.dequantize_blocks(flat))


def _case(seed, n, din, dout, k, dtype, empty=0.1, pad=0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    t = lambda *s: torch.randn(*s, generator=g, device=DEV)
    spread = torch.exp(t(din + pad))
    ids = torch.randint(0, k, (n,), generator=g, device=DEV)
    ids = torch.where(torch.rand(n, generator=g, device=DEV) < empty, -1, ids).to(torch.int32)
    W = km.quantize_blocks((t(k, dout, din) * torch.exp(t(k, dout, 1))).to(dtype))
    return {"X": (t(n, din + pad) * spread).to(dtype)[:, :din], "W": W, "ids": ids}


def _dropped(x, w, xe, we):
    """[rows, cols]: the most that the 8-bit instructions drop, 2^-10 2^m over groups of 8."""
    # 2^e <= |v|, -6 for subnormal values and zero
    e = lambda v: torch.where(v == 0, -5, torch.frexp(v)[1].clamp_min(-5)).to(F64) - 1
    pad = -x.shape[1] % 8
    x, w = (torch.nn.functional.pad(v, (0, pad)) for v in (x, w))
    out = torch.zeros(len(x), len(w), dtype=F64, device=DEV)
    for at in range(0, x.shape[1], 8):
        m = (e(x[:, None, at:at + 8]) + e(w[None, :, at:at + 8])).amax(2)
        power = xe[:, at // 128].int()[:, None] + we[:, at // 128].int()[None, :] - 254
        out += torch.exp2(m + power - 10)
    return out


def _run(c, dtype=None):
    k, dout, din = c["W"].shape
    q = km.quantize_blocks(c["X"])
    X, W = _stands(q), _stands(c["W"])
    plan = km.cluster_sort(c["ids"], k)
    y = km.cluster_linear_fp8(c["X"], c["W"], plan, dtype=dtype)
    t = dtype or c["X"].dtype
    assert y.dtype == t and y.shape == (len(X), dout)
    want, tol = torch.zeros(2, len(X), dout, dtype=F64, device=DEV)
    for i in range(k):
        at = torch.nonzero(c["ids"] == i)[:, 0]
        if len(at):
            want[at], tol[at] = X[at] @ W[i].T, 2 * din * u * (X[at].abs() @ W[i].abs().T)
            if t != torch.float32:
                tol[at] += 1.001 * _dropped(q.values[at].float(), c["W"].values[i].float(), q.exponents[at],
                                            c["W"].exponents[i])
    off = (y.to(F64) - want).abs() - tol - U[t] * want.abs() - (2.0 ** -25 if t == torch.float16 else 0)
    assert (off <= 0).all(), "off by %.3g over its tolerance" % float(off.max())
    assert torch.equal(km.cluster_linear_fp8(q, c["W"], plan, dtype=t), y)
    at = plan.order.long()
    assert torch.equal(km.cluster_linear_fp8(c["X"][at], c["W"], plan, sorted_rows=True, dtype=t), y[at])
    return y


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [1, 2, 17, 48, 64, 65, 200, 1000])
@pytest.mark.parametrize("din,dout,k", [(16, 16, 3), (128, 64, 1), (256, 320, 40), (250, 130, 7), (33, 47, 100),
                                        (1024, 512, 9), (400, 1001, 5)])
def test_rows(n, din, dout, k, dtype):
    print("case", n, din, dout, k, dtype, flush=True)
    _run(_case(n * 7 + k, n, din, dout, k, dtype))


@pytest.mark.parametrize("din", [1, 2, 15, 16, 17, 63, 64, 112, 127, 128, 129, 144, 256, 272, 385])
def test_widths(din):
    for n, dout in ((5, din + 3), (150, 64), (130, 72)):
        _run(_case(din, n, din, dout, 4, torch.bfloat16))


@pytest.mark.parametrize("n,din,dout,k", [(4200, 128, 4096, 5), (4097, 320, 1024, 8), (4500, 1000, 1100, 30),
                                          (2050, 4352, 2304, 3), (300, 8336, 200, 3), (20, 8448, 100, 3),
                                          (3000, 4357, 515, 3)])
def test_larger_tiles(n, din, dout, k):
    """Wider tiles, and contractions of more blocks than the scales that a tile holds at once."""
    print("case", n, din, dout, k, flush=True)
    c = _case(n, n, din, dout, k, torch.bfloat16)
    _run(c, torch.float32)
    _run(c)


def test_sizes_of_clusters():
    sizes = [3000, 256, 257, 0, 1, 255, 64, 65, 0, 63, 512, 513]
    ids = torch.repeat_interleave(torch.arange(len(sizes), device=DEV), torch.tensor(sizes, device=DEV))
    for din, dout in ((96, 72), (512, 2560)):
        c = _case(5, len(ids), din, dout, len(sizes), torch.bfloat16)
        c["ids"] = ids[torch.randperm(len(ids), device=DEV)].to(torch.int32).contiguous()
        _run(c)


def test_strided_rows():
    for pad in (16, 3):
        for n in (20, 333):
            _run(_case(pad, n, 64, 128, 5, torch.float16, pad=pad))


def test_nonfinite_values_stay_in_their_rows():
    for n, dout in ((30, 96), (3000, 2048)):
        c = _case(9, n, 256, dout, 4, torch.bfloat16, empty=0.0)
        y = _run(c)
        c["X"][5, 7], c["X"][n - 1, 200] = float("nan"), float("inf")
        plan = km.cluster_sort(c["ids"], 4)
        y2 = km.cluster_linear_fp8(c["X"], c["W"], plan)
        ok = torch.ones(n, dtype=torch.bool, device=DEV)
        ok[5] = ok[n - 1] = False
        assert torch.equal(y2[ok], y[ok]) and y2[~ok].isnan().all()


def test_no_rows_and_no_cluster():
    c = _case(1, 0, 64, 32, 4, torch.bfloat16)
    assert km.cluster_linear_fp8(c["X"], c["W"], km.cluster_sort(c["ids"], 4)).shape == (0, 32)
    for n in (3, 300):
        assert (_run(_case(1, n, 64, 64, 4, torch.bfloat16, empty=1.1)) == 0).all()


@pytest.mark.parametrize("n", [24, 700])
def test_side_stream_graph_and_repeats(n):
    c = _case(n, n, 384, 192, 6, torch.bfloat16)

    def step(stream=None):
        plan = km.cluster_sort(c["ids"], 6, stream=stream)
        q = km.quantize_blocks(c["X"], stream=stream)
        return (km.cluster_linear_fp8(c["X"], c["W"], plan, stream=stream),
                km.cluster_linear_fp8(q, c["W"], plan, stream=stream), km.dequantize_blocks(q, stream=stream))
    want = step()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step()
    for trial in range(3):
        c["X"].mul_(-0.7)
        c["ids"].copy_((c["ids"] + 1).clamp_max(5))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, step())), trial


def test_refusals():
    c = _case(1, 10, 200, 16, 4, torch.bfloat16, empty=0.0)
    X, W, ids = c["X"], c["W"], c["ids"]
    plan = km.cluster_sort(ids, 4)
    q = km.quantize_blocks(X)
    B = km.BlockRows
    for bad in (dict(X=X[:9]), dict(X=X.double()), dict(X=X[:, :190]), dict(X=X.cpu()), dict(W=B(W.values[0], W.exponents[0])),
                dict(W=B(W.values, W.exponents[:, :, :1])), dict(W=B(W.values, W.exponents.int())),
                dict(W=B(W.values.view(torch.uint8), W.exponents)), dict(W=B(W.values[:, :, :128], W.exponents)),
                dict(X=B(q.values, q.exponents[:9])), dict(X=B(q.values[:, :128], q.exponents[:, :1])),
                dict(plan=km.cluster_sort(ids, 5)), dict(dtype=torch.float64)):
        with pytest.raises(ValueError):
            km.cluster_linear_fp8(**dict(dict(X=X, W=W, plan=plan), **bad))
    for bad in (dict(W=W.values), dict(plan=ids)):
        with pytest.raises(TypeError):
            km.cluster_linear_fp8(**dict(dict(X=X, W=W, plan=plan), **bad))
    for bad in (X.double(), X.cpu(), X.t(), X[0], torch.zeros(2, 3, 4, device=DEV).transpose(1, 2)):
        with pytest.raises(ValueError):
            km.quantize_blocks(bad)
    with pytest.raises(ValueError):
        km.dequantize_blocks(q, torch.float64)
    with pytest.raises(TypeError):
        km.dequantize_blocks(q.values)
    with pytest.raises(ValueError, match="requires a gradient"):
        km.quantize_blocks(X.clone().requires_grad_())
