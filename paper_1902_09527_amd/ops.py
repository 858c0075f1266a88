"""Operators of a layer conditioned on clusters (include/kmeans_ops.h).

The assignment of :func:`run` (or any int32 cluster ids) routes rows -- the
tokens of a model, embeddings -- to small experts of their clusters:

  cluster_sort, cluster_gather, cluster_combine, cluster_combine_backward
      rows sorted by cluster and back with weights, and the gradients;
  layernorm, layernorm_backward
      the normalisation in front of them;
  adapter_linear, adapter_linear_backward
      a shared projection with one low-rank adapter per cluster;
  cluster_linear, cluster_linear_backward
      products with one weight per cluster;
  quantize_blocks, dequantize_blocks, cluster_linear_fp8
      rows in 8 bits with a scale for each 128 elements, and their products
      with one weight per cluster;
  cluster_embedding, cluster_embedding_backward
      rows of a table by their ids (a vocabulary's, the clusters' own);
  global_norm, clip_global_norm
      the norm over many tensors, and scaling them to a limit of it.

As in :mod:`.kmeans`, this is argument marshalling only: tensors are checked
and handed to the kernels of ``libkmeans_mti.so``.  Rows are float32, bfloat16
or float16 matrices on a GPU whose last dimension is contiguous; their row
stride may be anything from the width up.  Every function takes ``stream``:
work and the memory of its results belong to that stream (default: the
current one); as with any tensor, wait for it before using results elsewhere.
Nothing synchronizes.

Gradients are calls of their own (``*_backward``); autograd records none of
these calls, so a tensor that requires a gradient is refused while grad mode is
on, and one with a forward-mode tangent wherever its tangent would be lost.  Call them under ``torch.no_grad()``, or in the forward and backward of a
``torch.autograd.Function``, which run without it.
"""
from __future__ import annotations

import array
import math
import operator
from typing import Optional, Sequence, Tuple

import torch
from torch.autograd import forward_ad

from . import _native as N

_TYPES = {torch.float32: N.KM_F32, torch.bfloat16: N.KM_BF16, torch.float16: N.KM_F16}

# Sizes go to the library as 32-bit numbers (rows as 64-bit ones), and ctypes keeps a
# larger one's low bits without an error: they are checked here.
_MOST = 2 ** 31 - 1
_MOST_COLUMNS = 2 ** 28


def _too_large(what: str, most: str) -> N.KMError:
    return N.KMError(N.KM_ERR_INVALID_ARG, what, "at most %s" % most)


def _gpu(t: torch.Tensor, name: str, device: Optional[torch.device] = None) -> None:
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.device.type != "cuda":
        raise ValueError("%s must be on a GPU device, got %s" % (name, t.device))
    if device is not None and t.device != device:
        raise ValueError("%s must be on %s, got %s" % (name, device, t.device))


def _rows(t: torch.Tensor, name: str, like: Optional[torch.Tensor] = None, n: Optional[int] = None,
          d: Optional[int] = None) -> int:
    """Check a matrix of rows; its row stride."""
    _gpu(t, name, like.device if like is not None else None)
    if t.dtype not in _TYPES:
        raise ValueError("%s must be float32, bfloat16 or float16, got %s" % (name, t.dtype))
    if like is not None and t.dtype != like.dtype:
        raise ValueError("%s must be %s, got %s" % (name, like.dtype, t.dtype))
    if t.dim() != 2:
        raise ValueError("%s must be 2-D" % name)
    rows, cols = t.shape
    if cols < 1:
        raise ValueError("%s must have at least one column" % name)
    if cols > _MOST_COLUMNS:
        raise _too_large("columns of %s" % name, "2^28")
    if n is not None and rows != n:
        raise ValueError("%s must have %d rows, got %d" % (name, n, rows))
    if d is not None and cols != d:
        raise ValueError("%s must have %d columns, got %d" % (name, d, cols))
    ld, step = t.stride()
    if cols > 1 and step != 1:
        raise ValueError("%s must have contiguous rows (last stride 1)" % name)
    if rows <= 1:
        return cols
    if ld < cols:
        raise ValueError("%s must have rows that do not overlap" % name)
    return ld


def _array(t: torch.Tensor, name: str, dtype: torch.dtype, shape: Tuple[int, ...], device: torch.device) -> None:
    if isinstance(t, torch.Tensor) and t.dtype is dtype and t.shape == shape and t.device == device \
            and t.is_contiguous():
        return
    _gpu(t, name, device)
    if t.dtype != dtype:
        raise ValueError("%s must be %s, got %s" % (name, dtype, t.dtype))
    if tuple(t.shape) != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, shape, tuple(t.shape)))
    raise ValueError("%s must be contiguous" % name)


def _p(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _not_followed(inputs: Sequence[Optional[torch.Tensor]]) -> None:
    """Refuse inputs that autograd would follow, backward or forward (whose tangents
    no_grad leaves, and the forward of an autograd.Function hides)."""
    if torch.is_grad_enabled():
        for t in inputs:
            if t is not None and t.requires_grad:
                raise ValueError("an input requires a gradient, and autograd does not follow this call: use "
                                 "torch.no_grad() or a torch.autograd.Function, and the *_backward functions")
    if getattr(forward_ad, "_current_level", 0) >= 0:   # a level is open
        for t in inputs:
            if t is not None and forward_ad.unpack_dual(t).tangent is not None:
                raise ValueError("an input has a forward-mode tangent, and autograd does not follow this call: use "
                                 "a torch.autograd.Function with a jvp of its own")


class _On:
    """The device and stream of one call: results and workspaces are allocated
    on that stream, and inputs made on another one are kept until it has
    used them.  Inputs that autograd would follow are refused."""

    __slots__ = ("device", "stream", "inputs", "ctx")

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream],
                 inputs: Tuple[Optional[torch.Tensor], ...]):
        _not_followed(inputs)
        self.device, self.stream, self.inputs, self.ctx = device, stream, inputs, None

    def __enter__(self) -> int:
        if self.stream is not None:
            if self.stream.device != self.device:
                raise ValueError("stream is on %s, the tensors on %s" % (self.stream.device, self.device))
            self.ctx = torch.cuda.stream(self.stream)
            self.ctx.__enter__()
            for t in self.inputs:
                if t is not None:
                    t.record_stream(self.stream)
            return self.stream.cuda_stream
        index = self.device.index
        if torch.cuda.current_device() != index:
            self.ctx = torch.cuda.device(index)
            self.ctx.__enter__()
        return torch._C._cuda_getCurrentRawStream(index)   # current_stream's Stream object costs 1 us

    def __exit__(self, *exc) -> None:
        if self.ctx is not None:
            self.ctx.__exit__(*exc)


def _workspace(nbytes: int, device: torch.device, where: str) -> torch.Tensor:
    """Device memory for one call (torch's allocator aligns to 512 bytes)."""
    if nbytes == 0:
        raise N.KMError(N.KM_ERR_INVALID_ARG, where)
    return torch.empty(nbytes, dtype=torch.uint8, device=device)


class ClusterPlan:
    """Rows' slots sorted by cluster (made by :func:`cluster_sort`).

    ``order`` (int32 [n m]): the slots i * m + j by cluster, empty slots last;
    ``pos`` (int32, the ids' shape): its inverse; ``sorted_ids`` (int32
    [n m]): the cluster of each sorted place, -1 for empty slots; ``offsets``
    (int32 [k + 1]): cluster c's places are offsets[c] .. offsets[c + 1].
    """

    __slots__ = ("order", "pos", "sorted_ids", "offsets", "n", "m", "k")

    def __init__(self, order: torch.Tensor, pos: torch.Tensor, sorted_ids: torch.Tensor, offsets: torch.Tensor,
                 n: int, m: int, k: int):
        self.order, self.pos, self.sorted_ids, self.offsets = order, pos, sorted_ids, offsets
        self.n, self.m, self.k = n, m, k

    @property
    def device(self) -> torch.device:
        return self.offsets.device


def cluster_sort(ids: torch.Tensor, k: int, stream: Optional[torch.cuda.Stream] = None) -> ClusterPlan:
    """Sort rows by cluster (kmeans_sort_plan).

    ids: int32 [n] or [n, m], the cluster(s) of each row (``run``'s
    assignment has m = 1); an id outside [0, k) marks an empty slot.  Stable:
    slots of a cluster keep their order.
    """
    _gpu(ids, "ids")
    if ids.dtype != torch.int32:
        raise ValueError("ids must be int32, got %s" % ids.dtype)
    if ids.dim() not in (1, 2) or (ids.dim() == 2 and ids.shape[1] < 1):
        raise ValueError("ids must be [n] or [n, m] with m >= 1")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    k = int(k)
    n, m = ids.shape[0], ids.shape[1] if ids.dim() == 2 else 1
    dev = ids.device
    lib = N.load()
    if not 1 <= k < 2 ** 31 - 1 or n * m >= 2 ** 31:
        raise N.KMError(N.KM_ERR_INVALID_ARG, "kmeans_sort_plan", "1 <= k < 2^31 - 1 and n m < 2^31 needed")
    with _On(dev, stream, (ids,)) as s:
        # The plan is one allocation: the workspace may be let go, the views share their memory.
        order, pos, sorted_ids, offsets = ids.new_empty(3 * n * m + k + 1).split((n * m, n * m, n * m, k + 1))
        pos = pos.view(ids.shape)
        ws = _workspace(lib.kmeans_sort_workspace_bytes(n, m, k), dev, "kmeans_sort_workspace_bytes")
        st = lib.kmeans_sort_plan(_p(ids), n, m, k, _p(order), _p(pos), _p(sorted_ids), _p(offsets), _p(ws),
                                  ws.numel(), s)
    N.check(st, "kmeans_sort_plan")
    return ClusterPlan(order, pos, sorted_ids, offsets, n, m, k)


def _plan(plan: ClusterPlan, device: torch.device) -> None:
    if not isinstance(plan, ClusterPlan):
        raise TypeError("plan must be a ClusterPlan (cluster_sort)")
    if plan.device != device:
        raise ValueError("plan is on %s, the rows on %s" % (plan.device, device))


def cluster_gather(X: torch.Tensor, plan: ClusterPlan, stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Rows in cluster order (kmeans_sort_gather): [n m, d], place s holding row
    order[s] // m of X; places of empty slots are zero.  Its gradient with
    respect to X is ``cluster_combine(dXs, plan)``."""
    ld = _rows(X, "X", n=plan.n if isinstance(plan, ClusterPlan) else None)
    _plan(plan, X.device)
    d = X.shape[1]
    with _On(X.device, stream, (X, plan.pos, plan.offsets)) as s:
        out = X.new_empty((plan.n * plan.m, d))
        st = N.load().kmeans_sort_gather(_p(X), ld, plan.n, plan.m, plan.k, d, _TYPES[X.dtype], _p(plan.pos),
                                         _p(plan.offsets), _p(out), s)
    N.check(st, "kmeans_sort_gather")
    return out


def cluster_combine(Z: torch.Tensor, plan: ClusterPlan, weights: Optional[torch.Tensor] = None,
                    stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Sorted rows back to their rows (kmeans_sort_combine): [n, d], row i the
    sum of weights[i, j] Z[pos[i, j]] over its slots in use (zero for a row
    with none).  weights: float32 of the ids' shape, or None (ones)."""
    ld = _rows(Z, "Z", n=plan.n * plan.m if isinstance(plan, ClusterPlan) else None)
    _plan(plan, Z.device)
    if weights is not None:
        _array(weights, "weights", torch.float32, tuple(plan.pos.shape), Z.device)
    d = Z.shape[1]
    with _On(Z.device, stream, (Z, plan.pos, plan.offsets, weights)) as s:
        out = Z.new_empty((plan.n, d))
        st = N.load().kmeans_sort_combine(_p(Z), ld, plan.n, plan.m, plan.k, d, _TYPES[Z.dtype], _p(plan.pos),
                                          _p(plan.offsets), _p(weights), _p(out), s)
    N.check(st, "kmeans_sort_combine")
    return out


def cluster_combine_backward(dY: torch.Tensor, Z: torch.Tensor, plan: ClusterPlan, weights: torch.Tensor,
                             stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """Gradients of ``cluster_combine(Z, plan, weights)``: (dZ [n m, d], zero
    rows for empty slots; dweights float32 of the ids' shape, zero for empty
    slots).  Without weights the gradient is ``cluster_gather(dY, plan)``."""
    ld = _rows(dY, "dY", n=plan.n if isinstance(plan, ClusterPlan) else None)
    _plan(plan, dY.device)
    d = dY.shape[1]
    ldz = _rows(Z, "Z", like=dY, n=plan.n * plan.m, d=d)
    _array(weights, "weights", torch.float32, tuple(plan.pos.shape), dY.device)
    with _On(dY.device, stream, (dY, Z, plan.pos, plan.offsets, weights)) as s:
        dz = dY.new_empty((plan.n * plan.m, d))
        dw = torch.empty_like(weights)
        st = N.load().kmeans_sort_combine_backward(_p(dY), ld, _p(Z), ldz, plan.n, plan.m, plan.k, d,
                                                   _TYPES[dY.dtype], _p(plan.pos), _p(plan.offsets), _p(weights),
                                                   _p(dz), _p(dw), s)
    N.check(st, "kmeans_sort_combine_backward")
    return dz, dw


def _params(X: torch.Tensor, **params: Optional[torch.Tensor]) -> int:
    """Check a norm's parameters (all float32, or all of the rows' type); 1 for float32."""
    given = [(name, t) for name, t in params.items() if t is not None]
    for name, t in given:
        _gpu(t, name, X.device)
        if t.dtype not in (torch.float32, X.dtype) or t.dtype != given[0][1].dtype:
            raise ValueError("weight and bias must both be float32 or both %s" % X.dtype)
        _array(t, name, t.dtype, (X.shape[1],), X.device)
    return int(not given or given[0][1].dtype == torch.float32)


def layernorm(X: torch.Tensor, weight: Optional[torch.Tensor] = None, bias: Optional[torch.Tensor] = None,
              eps: float = 1e-5, stream: Optional[torch.cuda.Stream] = None
              ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Layer norm of rows (kmeans_norm_forward): (Y of X's type, mean and rstd
    float32 [n], which :func:`layernorm_backward` reads).  weight, bias: [d]
    or None, float32 or X's type."""
    ld = _rows(X, "X")
    f32 = _params(X, weight=weight, bias=bias)
    n, d = X.shape
    with _On(X.device, stream, (X, weight, bias)) as s:
        y = X.new_empty((n, d))
        mean, rstd = torch.empty((2, n), dtype=torch.float32, device=X.device).unbind()
        st = N.load().kmeans_norm_forward(_p(X), ld, n, d, _TYPES[X.dtype], _p(weight), _p(bias), f32, float(eps),
                                          _p(y), _p(mean), _p(rstd), s)
    N.check(st, "kmeans_norm_forward")
    return y, mean, rstd


def layernorm_backward(dY: torch.Tensor, X: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor,
                       weight: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients of :func:`layernorm` (kmeans_norm_backward): (dX of X's type,
    dweight and dbias float32 [d], whatever the weight's type)."""
    ld = _rows(X, "X")
    n, d = X.shape
    ldy = _rows(dY, "dY", like=X, n=n, d=d)
    f32 = _params(X, weight=weight)
    _array(mean, "mean", torch.float32, (n,), X.device)
    _array(rstd, "rstd", torch.float32, (n,), X.device)
    lib = N.load()
    with _On(X.device, stream, (dY, X, mean, rstd, weight)) as s:
        dx = X.new_empty((n, d))
        dg, db = torch.empty((2, d), dtype=torch.float32, device=X.device).unbind()
        ws = _workspace(lib.kmeans_norm_workspace_bytes(n, d, _TYPES[X.dtype]), X.device,
                        "kmeans_norm_workspace_bytes")
        st = lib.kmeans_norm_backward(_p(dY), ldy, _p(X), ld, n, d, _TYPES[X.dtype], _p(mean), _p(rstd),
                                      _p(weight), f32, _p(dx), _p(dg), _p(db), _p(ws), ws.numel(), s)
    N.check(st, "kmeans_norm_backward")
    return dx, dg, db


def _adapters(X: torch.Tensor, W: torch.Tensor, A: torch.Tensor, B: torch.Tensor,
              scale: Optional[torch.Tensor]) -> Tuple[int, int, int, int]:
    """Check the weights of an adapter projection; (din, dout, k, r)."""
    for t, name, dims in ((W, "W", 2), (A, "A", 3), (B, "B", 3)):
        if not isinstance(t, torch.Tensor) or t.dim() != dims or t.numel() == 0:
            _gpu(t, name, X.device)
            raise ValueError("%s must be a non-empty %d-D tensor" % (name, dims))
    (dout, din), (k, r, _) = W.shape, A.shape
    if X.shape[1] != din:
        raise ValueError("X must have %d columns" % din)
    _array(W, "W", X.dtype, (dout, din), X.device)
    _array(A, "A", X.dtype, (k, r, din), X.device)
    _array(B, "B", X.dtype, (k, dout, r), X.device)
    if max(dout, k, r) > _MOST:
        raise _too_large("sizes of W, A and B", "2^31 - 1")
    if scale is not None:
        _array(scale, "scale", torch.float32, (k,), X.device)
    return din, dout, k, r


def _places(plan: ClusterPlan, n: int, k: int, device: torch.device, sorted_rows: bool) -> Optional[torch.Tensor]:
    """Check a plan for n rows; its order, or None where the rows are in it already."""
    _plan(plan, device)
    if plan.k != k:
        raise ValueError("plan has %d clusters, the weights have %d" % (plan.k, k))
    if plan.m != 1 and not sorted_rows:
        raise ValueError("a plan of m = %d slots a row needs sorted rows (cluster_gather)" % plan.m)
    if plan.n * plan.m != n:
        raise ValueError("plan has %d places, X %d rows" % (plan.n * plan.m, n))
    return None if sorted_rows else plan.order


def adapter_linear(X: torch.Tensor, W: torch.Tensor, A: torch.Tensor, B: torch.Tensor, clusters,
                   scale: Optional[torch.Tensor] = None, sorted_rows: bool = False,
                   stream: Optional[torch.cuda.Stream] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """A shared projection with one low-rank adapter per cluster
    (kmeans_adapter_forward): for a row x of cluster c, h = A[c] x and
    y = W x + scale[c] B[c] h; a row in no cluster has h = 0, y = W x.

    W [dout, din], A [k, r, din], B [k, dout, r] (r up to 128) and X are of
    one type; scale is float32 [k] or None (ones).  ``clusters``: int32 ids
    [n], or a :class:`ClusterPlan` (with ``sorted_rows``, X is in the plan's
    order: the output of :func:`cluster_gather`).  Returns (Y [n, dout],
    H [n, r]); :func:`adapter_linear_backward` reads H.
    """
    ld = _rows(X, "X")
    din, dout, k, r = _adapters(X, W, A, B, scale)
    n, dev = X.shape[0], X.device
    ids = order = sids = offsets = None
    if isinstance(clusters, ClusterPlan):
        order = _places(clusters, n, k, dev, sorted_rows)
        sids, offsets = clusters.sorted_ids, clusters.offsets
    else:
        if sorted_rows:
            raise ValueError("sorted rows need a plan")
        _array(clusters, "clusters", torch.int32, (n,), dev)
        ids = clusters
    lib = N.load()
    need = lib.kmeans_adapter_workspace_bytes(n, din, dout, k, r, _TYPES[X.dtype], 0)
    if need == 0 and r > 128:
        raise N.KMError(N.KM_ERR_UNSUPPORTED, "kmeans_adapter_forward", "adapters have a rank of at most 128")
    with _On(dev, stream, (X, W, A, B, ids, order, sids, offsets, scale)) as s:
        y, h = X.new_empty((n, dout)), X.new_empty((n, r))
        ws = _workspace(need, dev, "kmeans_adapter_workspace_bytes")
        st = lib.kmeans_adapter_forward(_p(X), ld, n, din, dout, k, r, _TYPES[X.dtype], _p(W), _p(A), _p(B),
                                        _p(scale), _p(ids), _p(order), _p(sids), _p(offsets), _p(y), _p(h),
                                        _p(ws), ws.numel(), s)
    N.check(st, "kmeans_adapter_forward")
    return y, h


def adapter_linear_backward(dY: torch.Tensor, X: torch.Tensor, H: torch.Tensor, W: torch.Tensor, A: torch.Tensor,
                            B: torch.Tensor, plan: ClusterPlan, scale: Optional[torch.Tensor] = None,
                            sorted_rows: bool = False, stream: Optional[torch.cuda.Stream] = None
                            ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gradients of :func:`adapter_linear` (kmeans_adapter_backward): (dX, dA,
    dB), of the rows' type; W is frozen."""
    ld = _rows(X, "X")
    din, dout, k, r = _adapters(X, W, A, B, scale)
    n, dev = X.shape[0], X.device
    ldy = _rows(dY, "dY", like=X, n=n, d=dout)
    _array(H, "H", X.dtype, (n, r), dev)
    order = _places(plan, n, k, dev, sorted_rows)
    lib = N.load()
    need = lib.kmeans_adapter_workspace_bytes(n, din, dout, k, r, _TYPES[X.dtype], 1)
    if need == 0 and r > 128:
        raise N.KMError(N.KM_ERR_UNSUPPORTED, "kmeans_adapter_backward", "adapters have a rank of at most 128")
    with _On(dev, stream, (dY, X, H, W, A, B, order, plan.sorted_ids, plan.offsets, scale)) as s:
        dx = X.new_empty((n, din))
        da, db = torch.empty_like(A), torch.empty_like(B)
        ws = _workspace(need, dev, "kmeans_adapter_workspace_bytes")
        st = lib.kmeans_adapter_backward(_p(dY), ldy, _p(X), ld, _p(H), n, din, dout, k, r, _TYPES[X.dtype], _p(W),
                                         _p(A), _p(B), _p(scale), _p(order), _p(plan.sorted_ids),
                                         _p(plan.offsets), _p(dx), _p(da), _p(db), _p(ws), ws.numel(), s)
    N.check(st, "kmeans_adapter_backward")
    return dx, da, db


def _experts(X: torch.Tensor, W: torch.Tensor) -> Tuple[int, int, int]:
    """Check the weights of a product by cluster; (din, dout, k)."""
    if not isinstance(W, torch.Tensor) or W.dim() != 3 or W.numel() == 0:
        _gpu(W, "W", X.device)
        raise ValueError("W must be a non-empty 3-D tensor")
    k, dout, din = W.shape
    if X.shape[1] != din:
        raise ValueError("X must have %d columns" % din)
    _array(W, "W", X.dtype, (k, dout, din), X.device)
    if max(dout, k) > _MOST:
        raise _too_large("sizes of W", "2^31 - 1")
    return din, dout, k


def _linear_workspace(n: int, din: int, dout: int, k: int, type_: int, backward: int) -> int:
    need = N.load().kmeans_linear_workspace_bytes(n, din, dout, k, type_, backward)
    if need == 0:
        raise N.KMError(N.KM_ERR_UNSUPPORTED, "kmeans_linear_workspace_bytes",
                        "up to 2^27 rows, 2^24 columns and 2^31 tiles of 64 rows and columns")
    return need


def cluster_linear(X: torch.Tensor, W: torch.Tensor, plan: ClusterPlan, sorted_rows: bool = False,
                   stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Products with one weight per cluster (kmeans_linear_forward): y = W[c] x
    for a row x of cluster c, zeros for a row in no cluster; [n, dout].

    W [k, dout, din] and X are of one type.  ``plan``: a plan of one slot a row
    (``cluster_sort`` of [n] ids), or, with ``sorted_rows``, any plan in whose
    order X is (the output of :func:`cluster_gather`); results come in X's order.
    """
    ld = _rows(X, "X")
    din, dout, k = _experts(X, W)
    n, dev = X.shape[0], X.device
    order = _places(plan, n, k, dev, sorted_rows)
    need = _linear_workspace(n, din, dout, k, _TYPES[X.dtype], 0)
    with _On(dev, stream, (X, W, order, plan.sorted_ids, plan.offsets)) as s:
        y = X.new_empty((n, dout))
        ws = _workspace(need, dev, "kmeans_linear_workspace_bytes")
        st = N.load().kmeans_linear_forward(_p(X), ld, n, din, dout, k, _TYPES[X.dtype], _p(W), _p(order),
                                            _p(plan.sorted_ids), _p(plan.offsets), _p(y), _p(ws), ws.numel(), s)
    N.check(st, "kmeans_linear_forward")
    return y


def cluster_linear_backward(dY: torch.Tensor, X: torch.Tensor, W: torch.Tensor, plan: ClusterPlan,
                            sorted_rows: bool = False, need_dX: bool = True, need_dW: bool = True,
                            stream: Optional[torch.cuda.Stream] = None
                            ) -> Tuple[Optional[torch.Tensor], Optional[torch.Tensor]]:
    """Gradients of :func:`cluster_linear` (kmeans_linear_backward): (dX, dW), of
    the rows' type; zeros for rows in no cluster and clusters with no rows.  One
    that is not needed (``need_dX``, ``need_dW``) is None and not computed."""
    ld = _rows(X, "X")
    din, dout, k = _experts(X, W)
    n, dev = X.shape[0], X.device
    ldy = _rows(dY, "dY", like=X, n=n, d=dout)
    order = _places(plan, n, k, dev, sorted_rows)
    need = _linear_workspace(n, din, dout, k, _TYPES[X.dtype], 1)
    with _On(dev, stream, (dY, X, W, order, plan.offsets)) as s:
        dx = X.new_empty((n, din)) if need_dX else None
        dw = torch.empty_like(W) if need_dW else None
        ws = _workspace(need, dev, "kmeans_linear_workspace_bytes")
        st = N.load().kmeans_linear_backward(_p(dY), ldy, _p(X), ld, n, din, dout, k, _TYPES[X.dtype], _p(W), _p(order),
                                             _p(plan.offsets), _p(dx), _p(dw), _p(ws), ws.numel(), s)
    N.check(st, "kmeans_linear_backward")
    return dx, dw


_E4M3 = torch.float8_e4m3fn


class BlockRows:
    """Rows in 8-bit floating point (made by :func:`quantize_blocks`).

    ``values`` (float8_e4m3fn [..., d]) and ``exponents`` (uint8 [...,
    ceil(d / 128)]): 128 elements stand for values * 2^(exponent - 127), for
    NaN where the exponent is 255 (which is never made).
    """

    __slots__ = ("values", "exponents")

    def __init__(self, values: torch.Tensor, exponents: torch.Tensor):
        self.values, self.exponents = values, exponents

    @property
    def shape(self) -> torch.Size:
        return self.values.shape


def _blocks(q: BlockRows, name: str, dims: Tuple[int, ...], device: Optional[torch.device] = None) -> None:
    if not isinstance(q, BlockRows):
        raise TypeError("%s must be BlockRows (quantize_blocks)" % name)
    _gpu(q.values, name + ".values", device)
    if q.values.dim() not in dims or q.values.shape[-1] < 1:
        raise ValueError("%s must have %s dimensions and at least one column" % (name, " or ".join(map(str, dims))))
    shape = tuple(q.values.shape)
    if shape[-1] > _MOST_COLUMNS:
        raise _too_large("columns of %s" % name, "2^28")
    _array(q.values, name + ".values", _E4M3, shape, q.values.device)
    _array(q.exponents, name + ".exponents", torch.uint8, shape[:-1] + ((shape[-1] + 127) // 128,), q.values.device)


def quantize_blocks(X: torch.Tensor, stream: Optional[torch.cuda.Stream] = None) -> BlockRows:
    """Rows in 8 bits (kmeans_fp8_quantize): for each 128 elements of a row the
    least power of two under which none is beyond 448, and the values divided by
    it, rounded to e4m3; infinities and NaN become NaN.  X: rows [n, d], or
    contiguous [k, rows, d] (the weights of clusters)."""
    if isinstance(X, torch.Tensor) and X.dim() == 3:
        if not X.is_contiguous():
            raise ValueError("X must be contiguous")
        rows = X.view(X.shape[0] * X.shape[1], X.shape[2])
    else:
        rows = X
    ld = _rows(rows, "X")
    n, d = rows.shape
    with _On(X.device, stream, (X,)) as s:
        values = torch.empty(X.shape, dtype=_E4M3, device=X.device)
        exps = torch.empty(X.shape[:-1] + ((d + 127) // 128,), dtype=torch.uint8, device=X.device)
        st = N.load().kmeans_fp8_quantize(_p(rows), ld, n, d, _TYPES[X.dtype], _p(values), _p(exps), s)
    N.check(st, "kmeans_fp8_quantize")
    return BlockRows(values, exps)


def dequantize_blocks(Q: BlockRows, dtype: torch.dtype = torch.float32,
                      stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The values that ``Q`` stands for (kmeans_fp8_dequantize), of Q's shape."""
    _blocks(Q, "Q", (2, 3))
    if dtype not in _TYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16, got %s" % dtype)
    d, dev = Q.shape[-1], Q.values.device
    with _On(dev, stream, (Q.values, Q.exponents)) as s:
        out = torch.empty(Q.shape, dtype=dtype, device=dev)
        st = N.load().kmeans_fp8_dequantize(_p(Q.values), _p(Q.exponents), out.numel() // d, d, _TYPES[dtype], _p(out),
                                            s)
    N.check(st, "kmeans_fp8_dequantize")
    return out


def cluster_linear_fp8(X, W: BlockRows, plan: ClusterPlan, sorted_rows: bool = False,
                       dtype: Optional[torch.dtype] = None, stream: Optional[torch.cuda.Stream] = None
                       ) -> torch.Tensor:
    """:func:`cluster_linear` with both operands in 8 bits (kmeans_fp8_forward).

    W: [k, dout, din], quantised once.  X: rows [n, din], quantised in the call
    as :func:`quantize_blocks` does, or :class:`BlockRows`.  ``dtype``: of the
    results (default: X's type, bfloat16 for BlockRows).  For serving: the
    gradients of such a layer are those of :func:`cluster_linear`.

    float32 results have float32 sums.  For bfloat16 and float16 the matrix cores
    drop, of the products of each 8 consecutive elements, what lies more than 13
    bits below the largest one's exponent m (less than 2^-10 2^m of the 8 together)
    and add these sums in float32: 1.3e-5 of the norm for normal values, but up to
    two roundings of a float16 result where one product of 8 is far larger than the
    rest.  Where that counts, take float32 results and round them.
    """
    _blocks(W, "W", (3,))
    k, dout, din = W.shape
    dev = W.values.device
    if isinstance(X, BlockRows):
        _blocks(X, "X", (2,), dev)
        rows, exps, ld, kind = X.values, X.exponents, X.shape[1], N.KM_E4M3
    else:
        ld = _rows(X, "X")
        _gpu(X, "X", dev)
        rows, exps, kind = X, None, _TYPES[X.dtype]
    n = rows.shape[0]
    if rows.shape[1] != din or k < 1 or dout < 1:
        raise ValueError("X must have %d columns, and W weights" % din)
    if max(dout, k) > _MOST:
        raise _too_large("sizes of W", "2^31 - 1")
    dtype = dtype if dtype is not None else torch.bfloat16 if exps is not None else X.dtype
    if dtype not in _TYPES:
        raise ValueError("dtype must be float32, bfloat16 or float16, got %s" % dtype)
    order = _places(plan, n, k, dev, sorted_rows)
    lib = N.load()
    need = lib.kmeans_fp8_workspace_bytes(n, din, dout, k, kind)
    if need == 0:
        raise N.KMError(N.KM_ERR_UNSUPPORTED, "kmeans_fp8_workspace_bytes",
                        "up to 2^27 rows, 2^24 columns and 2^31 tiles of 64 rows and columns")
    with _On(dev, stream, (rows, exps, W.values, W.exponents, order, plan.sorted_ids, plan.offsets)) as s:
        y = torch.empty((n, dout), dtype=dtype, device=dev)
        ws = _workspace(need, dev, "kmeans_fp8_workspace_bytes")
        st = lib.kmeans_fp8_forward(_p(rows), ld, _p(exps), n, din, dout, k, kind, _p(W.values), _p(W.exponents),
                                    _p(order), _p(plan.sorted_ids), _p(plan.offsets), _p(y), _TYPES[dtype], _p(ws),
                                    ws.numel(), s)
    N.check(st, "kmeans_fp8_forward")
    return y


def _scale(scale: float) -> float:
    scale = float(scale)
    if not math.isfinite(scale):
        raise ValueError("scale must be finite")
    return scale


def cluster_embedding(ids: torch.Tensor, table: torch.Tensor, scale: float = 1.0,
                      stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Rows of a table by their ids (kmeans_table_forward): scale * table[id] for
    each of the ids (int32, any shape: tokens, or ``run``'s assignment), zeros
    for an id outside [0, k); of shape ids.shape + (d,).  table: rows [k, d]."""
    ld = _rows(table, "table")
    k, d = table.shape
    _gpu(ids, "ids", table.device)
    if k < 1:
        raise ValueError("table must have at least one row")
    if k > _MOST:
        raise _too_large("rows of table", "2^31 - 1")
    _array(ids, "ids", torch.int32, tuple(ids.shape), table.device)
    scale = _scale(scale)
    with _On(table.device, stream, (ids, table)) as s:
        y = table.new_empty(ids.shape + (d,))
        st = N.load().kmeans_table_forward(_p(ids), ids.numel(), k, d, _TYPES[table.dtype], _p(table), ld, scale, _p(y),
                                           s)
    N.check(st, "kmeans_table_forward")
    return y


def cluster_embedding_backward(dY: torch.Tensor, plan: ClusterPlan, scale: float = 1.0,
                               stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Gradient of :func:`cluster_embedding` for its table (kmeans_table_backward):
    [k, d] of dY's type, scale times the sum of dY over each id's slots, zeros
    for an id without any.  plan: ``cluster_sort(ids, k)``; dY: rows [n m, d], one
    for each slot.  Sums are float32 and do not depend on the run."""
    ld = _rows(dY, "dY", n=plan.n * plan.m if isinstance(plan, ClusterPlan) else None)
    _plan(plan, dY.device)
    n, d = dY.shape
    scale = _scale(scale)
    lib = N.load()
    with _On(dY.device, stream, (dY, plan.order, plan.sorted_ids, plan.offsets)) as s:
        out = dY.new_empty((plan.k, d))
        ws = _workspace(lib.kmeans_table_workspace_bytes(n, plan.k, d, _TYPES[dY.dtype]), dY.device,
                        "kmeans_table_workspace_bytes")
        st = lib.kmeans_table_backward(_p(dY), ld, n, plan.k, d, _TYPES[dY.dtype], _p(plan.order), _p(plan.sorted_ids),
                                       _p(plan.offsets), scale, _p(out), _p(ws), ws.numel(), s)
    N.check(st, "kmeans_table_backward")
    return out


# A list of many small tensors costs the host more than the GPU (160 tensors: 100 us
# a call): what is asked of each is asked by map over the list, and no more than once.
_dtype, _grad = operator.attrgetter("dtype"), operator.attrgetter("requires_grad")


def _tensors(tensors: Sequence[torch.Tensor], name: str) -> Tuple[list, array.array, list]:
    """Check a list of contiguous tensors; (tensors, sizes, dtypes).  That all are on
    the first one's device is checked with their addresses, in the call."""
    given = list(tensors)
    if not given:
        raise ValueError("%s: at least one is needed" % name)
    try:
        dense = all(map(torch.Tensor.is_contiguous, given))
    except TypeError:
        raise TypeError("%s must be torch.Tensors" % name) from None
    if not dense:
        raise ValueError("%s must be contiguous" % name)
    if not given[0].is_cuda:
        raise ValueError("%s must be on one GPU device" % name)
    dtypes = list(map(_dtype, given))
    if dtypes[0] not in _TYPES or (dtypes.count(dtypes[0]) != len(dtypes) and not set(dtypes) <= _TYPES.keys()):
        raise ValueError("%s must be float32, bfloat16 or float16" % name)
    return given, array.array("q", map(torch.Tensor.numel, given)), dtypes


def _clip(tensors: Sequence[torch.Tensor], limit: float, out: Optional[Sequence[torch.Tensor]], inplace: bool,
          stream: Optional[torch.cuda.Stream]) -> torch.Tensor:
    given, sizes, dtypes = _tensors(tensors, "tensors")
    dev, count = given[0].device, len(given)
    pointers = array.array("Q", map(torch.Tensor.data_ptr, given))
    to, targets = [], pointers if inplace else None
    if out is not None:
        to, to_sizes, to_dtypes = _tensors(out, "out")
        if to_sizes != sizes or to_dtypes != dtypes:
            raise ValueError("out must have the tensors' sizes and types")
        targets = array.array("Q", map(torch.Tensor.data_ptr, to))
    if (torch.is_grad_enabled() and (any(map(_grad, given)) or any(map(_grad, to)))) or \
            getattr(forward_ad, "_current_level", 0) >= 0:
        _not_followed(given + to)
    kinds = array.array("i", [_TYPES[dtypes[0]]]) * count if dtypes.count(dtypes[0]) == count else \
        array.array("i", [_TYPES[t] for t in dtypes])
    at = lambda a: None if a is None else a.buffer_info()[0]
    lib = N.load()
    with _On(dev, stream, tuple(given + to) if stream is not None else ()) as s:
        norm = torch.empty((), dtype=torch.float32, device=dev)
        ws = _workspace(lib.kmeans_clip_workspace_bytes(at(sizes), count), dev, "kmeans_clip_workspace_bytes")
        st = lib.kmeans_clip_norm(at(pointers), at(targets), at(sizes), at(kinds), count, limit, _p(norm), _p(ws),
                                  ws.numel(), s)
    if st != N.KM_OK and any(t.device != dev for t in given + to):
        raise ValueError("all tensors must be on %s" % dev)
    N.check(st, "kmeans_clip_norm")
    if targets is not None:
        torch.autograd.graph.increment_version(given if inplace else to)
    return norm


def global_norm(tensors: Sequence[torch.Tensor], stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """The square root of the sum of all squares over contiguous tensors of one
    device (kmeans_clip_norm), formed in float64: a float32 tensor of no
    dimensions (infinity beyond its range)."""
    return _clip(tensors, 1.0, None, False, stream)


def clip_global_norm(tensors: Sequence[torch.Tensor], limit: float, out: Optional[Sequence[torch.Tensor]] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> torch.Tensor:
    """Scale tensors so that their :func:`global_norm` is at most ``limit``
    (kmeans_clip_norm): each times min(1, limit / norm), in place, or to ``out``
    (tensors of the same sizes and types that overlap none of them).  Returns the
    norm before.  Where an input is infinite or NaN, the norm shows it and the values
    stay as they are; a norm beyond float32's range is returned as infinity and the
    values are scaled by the one in float64."""
    limit = float(limit)
    if not limit > 0:
        raise ValueError("limit must be positive")
    return _clip(tensors, limit, out, out is None, stream)
