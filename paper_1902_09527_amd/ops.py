"""Operators of a layer conditioned on clusters (include/kmeans_ops.h).

The assignment of :func:`run` (or any int32 cluster ids) routes rows -- the
tokens of a model, embeddings -- to small experts of their clusters:

  cluster_sort, cluster_gather, cluster_combine, cluster_combine_backward
      rows sorted by cluster and back with weights, and the gradients;
  layernorm, layernorm_backward
      the normalisation in front of them;
  adapter_linear, adapter_linear_backward
      a shared projection with one low-rank adapter per cluster.

As in :mod:`.kmeans`, this is argument marshalling only: tensors are checked
and handed to the kernels of ``libkmeans_mti.so``.  Rows are float32, bfloat16
or float16 matrices on a GPU whose last dimension is contiguous; their row
stride may be anything from the width up.  Every function takes ``stream``:
work and the memory of its results belong to that stream (default: the
current one); as with any tensor, wait for it before using results elsewhere.
Nothing synchronizes.

Gradients are calls of their own (``*_backward``); autograd records none of
these calls, so a tensor that requires a gradient is refused while grad mode is
on.  Call them under ``torch.no_grad()``, or in the forward and backward of a
``torch.autograd.Function``, which run without it.
"""
from __future__ import annotations

from typing import Optional, Tuple

import torch

from . import _native as N

_TYPES = {torch.float32: N.KM_F32, torch.bfloat16: N.KM_BF16, torch.float16: N.KM_F16}


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


class _On:
    """The device and stream of one call: results and workspaces are allocated
    on that stream, and inputs made on another one are kept until it has
    used them.  Inputs that autograd would follow are refused: it cannot."""

    __slots__ = ("device", "stream", "inputs", "ctx")

    def __init__(self, device: torch.device, stream: Optional[torch.cuda.Stream],
                 inputs: Tuple[Optional[torch.Tensor], ...]):
        if torch.is_grad_enabled():
            for t in inputs:
                if t is not None and t.requires_grad:
                    raise ValueError("an input requires a gradient, and autograd does not follow this call: use "
                                     "torch.no_grad() or a torch.autograd.Function, and the *_backward functions")
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
        return torch.cuda.current_stream(index).cuda_stream

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
    if scale is not None:
        _array(scale, "scale", torch.float32, (k,), X.device)
    return din, dout, k, r


def _places(plan: ClusterPlan, n: int, k: int, device: torch.device, sorted_rows: bool) -> Optional[torch.Tensor]:
    """Check a plan for n rows; its order, or None where the rows are in it already."""
    _plan(plan, device)
    if plan.k != k:
        raise ValueError("plan has %d clusters, A has %d" % (plan.k, k))
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
