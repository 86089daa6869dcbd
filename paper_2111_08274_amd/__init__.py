"""HADFL aggregation-cycle hot path for MI355X (gfx950).

``paper_2111_08274_amd.hadfl`` is the thin binding over the C-ABI library
``libhadfl.so`` (hand-written HIP kernels); ``paper_2111_08274_amd.synth`` holds
the seeded synthetic-input generators; ``next_token`` trains next-token heads on replicas with the operators of a language
model's head.  Importing the package loads none of them.
"""
__all__ = ["hadfl", "synth"]
