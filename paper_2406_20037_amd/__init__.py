"""MI355X (gfx950) implementation of the schedule-tuning hot path of the
combined Ansor + Droplet Search approach: a schedule-parameterised fp32
conv2d / matmul kernel family in HIP, a hipEvent measurement harness, a seeded
exploration sampler and Droplet Search coordinate descent, behind the C ABI
of ``include/droplet.h``; and the 8-bit operators of the same ABI (``Q8``,
``ds_q8_quantize``, ``ds_q8_matmul``, ``ds_swiglu8``, ``ds_swiglu8_grad``; ``Cache8``, ``Chunk``,
``ds_rotary``, ``ds_cache8_write``, ``ds_cache8_read``, ``ds_attn8``).
``_lib`` is the Python binding of that ABI; it is loaded on first use of any
name below, and raises if the library is missing.
"""
import sys
import types

_EXPORTS = ["Cache8", "Chunk", "DS_OP_CONV2D_NCHW", "DS_OP_MATMUL_RM", "Q8", "Space", "ansor_sample",
            "droplet_tune", "droplet_tune_ex", "ds_attn8", "ds_attn8_work", "ds_cache8_read",
            "ds_cache8_write", "ds_empty_kernel_floor", "ds_measure", "ds_q8_matmul", "ds_q8_quantize",
            "ds_rotary", "ds_swiglu8", "ds_swiglu8_grad", "ds_tune", "kernel_run",
            "kernel_run_reference", "make_io", "measure_cfg", "tune_cfg"]

__all__ = _EXPORTS + ["_lib"]


class _Name:
    """A name of the binding, looked up there at every use (a quarter of the time of a module's
    __getattr__, which a call of few microseconds notices)."""

    def __init__(self, name):
        self.name = name

    def __get__(self, package, kind=None):
        return getattr(package._lib, self.name)


class _Package(types.ModuleType):
    pass


for _name in _EXPORTS:
    setattr(_Package, _name, _Name(_name))
sys.modules[__name__].__class__ = _Package


def __getattr__(name):
    if name == "_lib":                   # the import binds it here
        import importlib
        return importlib.import_module("._lib", __name__)
    raise AttributeError(name)
