"""Composed affine copies on B200: compose a chain of layout operators into one
affine access map on the host and run it as a single CUDA copy kernel.

The CUDA/C++ library is loaded lazily by `paper_2002_12798_b200.binding`;
`paper_2002_12798_b200.workloads` (plain data) imports without it.  `paper_2002_12798_b200.ops` has the operators on
split heads whose addresses depend on data: rotary positions, a paged cache (16, 8 or 4 bits), its attention, and sampling.
"""
__all__ = ["binding", "ops", "workloads"]
