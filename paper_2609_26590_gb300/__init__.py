"""GB300-native chunkwise gated-linear-attention forward (the GTR token mixer).

The compute path is a C-ABI shared library of hand-written sm_103a CUDA
kernels (``csrc/``, declared in ``include/gtr_gla.h``); :mod:`.gla` is the thin
ctypes binding over it and uses PyTorch only for device memory and streams; it
also holds the operators around the mixer (layer norm, causal convolution,
selective scan, gated feed-forward step and the backward passes).
:mod:`.workloads` draws the seeded synthetic inputs.
"""
__all__ = ["gla", "workloads"]
