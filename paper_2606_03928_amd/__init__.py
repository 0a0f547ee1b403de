"""VaSE-AttnV eviction round for AMD Instinct MI355X (gfx950).

``vase`` is the binding of the HIP library ``libvase.so`` (built in-tree by
``paper_2606_03928_amd.build``); ``synth`` draws the synthetic Qwen3-shaped
caches; ``pages`` is the paged cache.  The library is loaded on first use, so
importing the package does not need a GPU.
"""
from . import pages, synth, vase  # noqa: F401

__all__ = ["pages", "synth", "vase"]
