"""MI355X-native ES parameter path: seeded perturb / restore / fused update /
reward z-score over lists of bf16 tensors (arXiv 2608.17310, Section 3).

Beside it stands what scores a member between two moves of the parameters: a
paged cache of keys and values, the attention over it (``kvcache``), the
log-probabilities and divergences at a decoder's head with their gradients
(``head``), projections under the low-rank adapters of many members
(``adapters``) and a decoder that evaluates the plan's parameters in place
(``rollout``).

The compute runs in the HIP library ``libesopt.so`` (csrc/); ``esopt`` is its
thin ctypes binding.  Importing this package does not load the library; the
first call into ``esopt`` does, and fails loudly if it has not been built.
"""

__all__ = ["esopt", "workloads", "kvcache", "head", "adapters", "rollout"]
