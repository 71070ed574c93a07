"""GB300 (sm_103a) SpGEMM: C = A*B for CSR matrices, computed by hand-written CUDA kernels;
also the elementwise operations C = A + B and C = A .* B and the sparse
matrix - sparse vector product y = A x, and the operations of layers that send
rows of dense matrices along a sparse routing matrix (``routing``).

The C ABI lives in include/ws_spgemm.h and libws_spgemm.so (built by
``paper_2606_20855_gb300.build``).  ``_abi`` is the ctypes binding with the
same function names; ``spgemm`` holds the PyTorch-facing wrapper.  Importing
this package loads nothing; the library is loaded on first use.
"""

__all__ = ["DeviceCSR", "SpGEMM", "SpGEMMOuter", "spgemm", "spgemm_outer", "submatrix", "Ewise", "ewise", "SpMSpV", "spmspv"]
_ROUTING = ["Routing", "topk_route", "topk_route_backward", "adapters"]
__all__ += _ROUTING


def __getattr__(name):
    if name not in __all__:
        raise AttributeError(name)
    import importlib
    m = importlib.import_module(f"{__name__}.{'routing' if name in _ROUTING else 'spgemm'}")
    globals()[name] = found = m if name == "spgemm" else getattr(m, name)  # that module, called, is its function of the same name
    return found
