"""Batched J-DOB policy evaluation on MI355X (gfx950).

The compute path is the C-ABI library ``libjdob.so`` built from
``csrc/jdob.hip``; ``paper_2504_14611_amd.jdob`` is its thin ctypes binding
and ``paper_2504_14611_amd.workloads`` generates seeded synthetic inputs.
``paper_2504_14611_amd.edge`` binds the edge operators (``edge_csrc/``), which
compute sub-tasks of a decoder network for the users that a policy offloads.
Importing the package loads nothing: the bindings load the library on first
use and raise if it is missing.
"""

__all__ = ["edge", "jdob", "workloads"]
