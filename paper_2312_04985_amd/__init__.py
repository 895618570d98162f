"""SparQ Attention decode step for one MI355X, and the paged cache that it starts from: hand-written HIP kernels behind a C ABI.

`binding` is the thin ctypes layer over libsparq.so (argument marshalling only),
`cache` and `paged` hold the buffers of a SparQ cache and of a cache in pages,
`workloads` draws the seeded synthetic inputs, `traffic` is the paper's transfer model.
Nothing here computes any part of the method on the host.
"""
__all__ = ["binding", "cache", "paged", "workloads", "traffic"]
