"""MI355X-native ZipLine barrier search (ElasticBSP, arXiv 2001.01347).

``workloads`` draws the seeded synthetic inputs; ``zipline`` is the thin ctypes
binding over the HIP library built from ``csrc/``, ``training`` that of the training
operators in the same library.  The binding loads the
library on first use and raises if it has not been built: there is no CPU
fallback.
"""
from . import workloads  # noqa: F401

__all__ = ["workloads", "zipline", "training"]


def __getattr__(name):
    if name in ("zipline", "training"):
        import importlib
        return importlib.import_module("." + name, __name__)
    raise AttributeError(name)
