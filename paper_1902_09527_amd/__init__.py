"""MI355X-native hot path of clusterNOR's k-means (arXiv 1902.09527).

Lloyd's k-means with Minimal Triangle Inequality pruning as hand-written HIP
kernels for gfx950 behind a C ABI (include/kmeans_mti.h); this package holds
the kernels (csrc/), the build step (build.py) and a thin ctypes binding.
ops.py holds the operators of a layer conditioned on clusters
(include/kmeans_ops.h).
"""
from .kmeans import KMeansMTI, kmeanspp, kmeanspp_workspace_bytes, run, run_pp_best  # noqa: F401
from .ops import (ClusterPlan, adapter_linear, adapter_linear_backward, cluster_combine,  # noqa: F401
                  cluster_combine_backward, cluster_gather, cluster_sort, layernorm, layernorm_backward)

__all__ = ["KMeansMTI", "kmeanspp", "kmeanspp_workspace_bytes", "run", "run_pp_best",
           "ClusterPlan", "cluster_sort", "cluster_gather", "cluster_combine", "cluster_combine_backward",
           "layernorm", "layernorm_backward", "adapter_linear", "adapter_linear_backward"]
