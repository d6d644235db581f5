"""MI355X-native cached mixed-precision EmbeddingBag training step.

The compute path lives in HIP kernels behind the C ABI declared in
``include/emb_cache.h`` (library ``paper_2010_11305_amd/libembcache.so``);
``paper_2010_11305_amd.emb_cache`` is the thin ctypes binding.  ``mx4``, ``adamw``,
``rmsnorm``, ``w4`` and ``clip`` bind the dense operators of ``include/emb_dense.h`` in the same library, and ``tower``
trains a model on both.  Importing this package loads nothing; the bindings load the
library on first use and raise if it has not been built.
"""
__all__ = ["configs", "workload", "emb_cache", "mx4", "adamw", "rmsnorm", "w4", "clip", "tower"]
