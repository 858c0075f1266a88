"""MI355X-native hot path of clusterNOR's k-means (arXiv 1902.09527).

Lloyd's k-means with Minimal Triangle Inequality pruning as hand-written HIP
kernels for gfx950 behind a C ABI (include/kmeans_mti.h); this package holds
the kernels (csrc/), the build step (build.py) and a thin ctypes binding.
ops.py holds the operators of a layer conditioned on clusters
(include/kmeans_ops.h).
"""
from .kmeans import KMeansMTI, kmeanspp, kmeanspp_workspace_bytes, run, run_pp_best  # noqa: F401
from .ops import (BlockRows, ClusterPlan, adapter_linear, adapter_linear_backward, clip_global_norm,  # noqa: F401
                  cluster_combine, cluster_combine_backward, cluster_embedding, cluster_embedding_backward,
                  cluster_gather, cluster_linear, cluster_linear_backward, cluster_linear_fp8, cluster_sort,
                  dequantize_blocks, global_norm, layernorm, layernorm_backward, quantize_blocks)

__all__ = ["KMeansMTI", "kmeanspp", "kmeanspp_workspace_bytes", "run", "run_pp_best",
           "ClusterPlan", "cluster_sort", "cluster_gather", "cluster_combine", "cluster_combine_backward",
           "layernorm", "layernorm_backward", "adapter_linear", "adapter_linear_backward",
           "cluster_linear", "cluster_linear_backward",
           "BlockRows", "quantize_blocks", "dequantize_blocks", "cluster_linear_fp8",
           "cluster_embedding", "cluster_embedding_backward", "global_norm", "clip_global_norm"]
