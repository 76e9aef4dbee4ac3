"""MI355X-native stage-boundary codec of AQ-SGD (activation-change quantisation), and the products of 8-bit
matrices that a stage makes on either side of a boundary.

``paper_2206_01299_amd.binding`` is the thin ctypes layer over the C-ABI
library built from ``csrc/``; ``paper_2206_01299_amd.workloads`` draws the
seeded synthetic inputs.  Importing the package loads nothing native.
"""
__all__ = ["binding", "workloads", "build"]
