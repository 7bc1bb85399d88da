"""RheoSampling draft-tree sampling and verification on one GB300 (sm_103a).

The compute lives in ``librheo.so`` (hand-written CUDA, C ABI in
``include/rheo.h``); ``rheo`` is its ctypes binding and ``synth`` the seeded
synthetic workloads.  Build the library with ``build.build()``.
"""
from .rheo import (CacheConfig, CachePlan, CacheWorkspace, Config, LogprobConfig, Logprobs, LogprobWorkspace, Pages,
                   Pruned, RheoError, Tree, TreeAttn, VerifyOut, Workspace, cache_commit, cache_reserve, expand,
                   library_path, make_cache, prune, qk_norm_rope, scratch_status, status, token_logprobs, tree_attend,
                   tree_attention, verify)

__all__ = ["Config", "Tree", "Pruned", "VerifyOut", "Workspace", "expand", "prune", "verify", "status",
           "RheoError", "library_path", "CacheConfig", "CachePlan", "CacheWorkspace", "LogprobConfig", "Logprobs",
           "LogprobWorkspace", "Pages", "TreeAttn", "cache_commit", "cache_reserve", "make_cache", "qk_norm_rope",
           "scratch_status", "token_logprobs", "tree_attend", "tree_attention"]
