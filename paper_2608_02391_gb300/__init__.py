"""GB300-native CoPES evolution-strategy core.

The compute lives in the CUDA library ``libcopes.so`` (built from ``csrc/`` for sm_103a);
``copes`` is its thin ctypes binding, ``es`` holds the schedules, ``rollout`` a decoder that
answers with the weights under evolution, and ``workloads`` describes the seeded synthetic
workloads.  Importing the package does not load the library; ``copes.load()`` (called by
every binding function) does, and raises if it is missing.
"""
__all__ = ["copes", "es", "rollout", "workloads"]
