"""B200 (sm_100a) allowed-token mask build + apply for operator-automaton structured decoding.

The product is the C-ABI library ``libwg.so`` (``include/wg.h``); this package is its thin
Python binding.  Build the library with ``python -m paper_2507_16768_b200.build``.  The
binding is loaded on first use and raises ImportError if the library has not been built:
there is no CPU fallback.
"""
import importlib
import sys
import types

__all__ = ["build", "binding"]

_binding = None


class _Package(types.ModuleType):
    """The package itself.  A name of the binding that has been asked for once becomes an attribute of this class,
    which costs a look-up a third of what ``__getattr__`` does (0.1 us instead of 0.3)."""


class _Name:
    """A name of the binding as it is there now: one that is replaced in the binding is replaced here."""

    def __init__(self, name):
        self.name = name

    def __get__(self, package, cls):
        return getattr(_binding, self.name)


def __getattr__(name):
    global _binding
    if name == "build":
        return importlib.import_module(".build", __name__)
    if _binding is None:
        _binding = importlib.import_module(".binding", __name__)
    if name == "binding":
        return _binding
    try:
        value = getattr(_binding, name)
    except AttributeError:
        raise AttributeError(f"module {__name__!r} has no attribute {name!r}") from None
    setattr(_Package, name, _Name(name))
    return value


sys.modules[__name__].__class__ = _Package
