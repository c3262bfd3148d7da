"""ctypes binding of ``libdroplet.so`` (argument marshalling only).

Every function here forwards to the C ABI declared in ``include/droplet.h``
under the same name.  Tensors may be passed as ``torch.Tensor`` (their
``data_ptr()`` is used) or as raw integer device addresses; streams as
``torch.cuda.Stream``, an integer ``hipStream_t`` or ``None`` (the current
torch stream when torch has a device, else the null stream).

The library must have been built (``paper_2406_20037_amd.build``); importing
this module without it raises, there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import os
import struct

try:
    # PyTorch ships its own HIP runtime (same soname).  Loading it before the
    # library makes the library bind to that runtime, so device pointers and
    # streams handed over from torch belong to the runtime the kernels use.
    import torch as _torch  # noqa: F401
except ImportError:  # plain C-ABI use without torch
    _torch = None

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libdroplet.so")

DS_OK = 0
DS_EINVAL = -1
DS_EUNSUPPORTED = -2
DS_EINVALID_SCHED = -3
DS_EHIP = -4
DS_EPARITY = -5
DS_EBUDGET = -6
DS_EEXHAUSTED = -7
DS_ENOMEM = -8
STATUS_NAMES = {0: "DS_OK", -1: "DS_EINVAL", -2: "DS_EUNSUPPORTED", -3: "DS_EINVALID_SCHED",
                -4: "DS_EHIP", -5: "DS_EPARITY", -6: "DS_EBUDGET", -7: "DS_EEXHAUSTED",
                -8: "DS_ENOMEM"}

DS_OP_CONV2D_NCHW = 1
DS_OP_MATMUL_RM = 2
DS_KERNEL_CONV_VALU, DS_KERNEL_CONV_MFMA, DS_KERNEL_MM_VALU, DS_KERNEL_MM_MFMA, DS_KERNEL_CONV_MFMA2 = 1, 2, 3, 4, 5
DS_MAX_KNOBS = 12
DS_MAX_REPEATS = 64
DS_NOALLOC_MAX_FLOATS = 8388608   # kernel_run_noalloc: split partials capacity


DS_TYPE_F32, DS_TYPE_F16, DS_TYPE_BF16 = 0, 1, 2
DS_Q8_E4M3, DS_Q8_E5M2 = 0, 1
DS_SCALE_POW2, DS_SCALE_F32 = 0, 1
DS_Q8_BLOCK = 128
DS_EXACT_SUMS = 256
DS_ROTARY_HALVES, DS_ROTARY_PAIRS, DS_ROTARY_INVERSE = 0, 1, 2


class ds_q8(C.Structure):
    _fields_ = [("data", C.c_void_p), ("scale", C.c_void_p), ("rows", C.c_int64),
                ("cols", C.c_int64), ("ld", C.c_int64), ("scale_ld", C.c_int64),
                ("format", C.c_int32), ("scale_type", C.c_int32), ("block_rows", C.c_int32),
                ("reserved", C.c_int32)]


class ds_heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("tokens", C.c_int64), ("heads", C.c_int64), ("dim", C.c_int64),
                ("ld", C.c_int64), ("head_ld", C.c_int64), ("type", C.c_int32), ("reserved", C.c_int32)]


class ds_cache8(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_scale", C.c_void_p), ("v_scale", C.c_void_p),
                ("pages", C.c_int64), ("stride", C.c_int64), ("scale_stride", C.c_int64),
                ("page", C.c_int32), ("heads", C.c_int32), ("dim", C.c_int32), ("format", C.c_int32),
                ("scale_type", C.c_int32), ("reserved", C.c_int32)]


class ds_chunk(C.Structure):
    _fields_ = [("starts", C.c_void_p), ("lengths", C.c_void_p), ("table", C.c_void_p),
                ("seqs", C.c_int64), ("table_cols", C.c_int64), ("table_ld", C.c_int64)]


class ds_attn8_cfg(C.Structure):
    _fields_ = [("scale", C.c_double), ("causal", C.c_int32), ("reserved", C.c_int32),
                ("window", C.c_int64), ("max_len", C.c_int64)]


class ds_sched(C.Structure):
    _fields_ = [("op", C.c_int32), ("nknobs", C.c_int32), ("shape", C.c_int64 * 9),
                ("idx", C.c_int32 * DS_MAX_KNOBS)]

    def index(self):
        return tuple(self.idx[a] for a in range(self.nknobs))


class ds_geometry(C.Structure):
    _fields_ = [("valid", C.c_int32), ("threads", C.c_int32), ("grid", C.c_int64),
                ("lds_bytes", C.c_int32), ("acc", C.c_int32), ("unroll_eff", C.c_int32),
                ("t0", C.c_int32), ("t1", C.c_int32), ("red", C.c_int32), ("chunks", C.c_int64)]


class ds_kernel_info(C.Structure):
    _fields_ = [("family", C.c_int32), ("nparams", C.c_int32), ("params", C.c_int32 * 6),
                ("instance", C.c_int32), ("threads", C.c_int32), ("grid", C.c_int64),
                ("lds_bytes", C.c_int32), ("splits", C.c_int32), ("args_hash", C.c_uint64),
                ("num_regs", C.c_int32), ("max_threads_per_block", C.c_int32),
                ("local_bytes", C.c_int64), ("static_lds_bytes", C.c_int64)]

    def as_dict(self):
        return {f: (list(getattr(self, f))[: self.nparams] if f == "params" else getattr(self, f))
                for f, _ in self._fields_}


class ds_measure_cfg(C.Structure):
    _fields_ = [("warmup", C.c_int32), ("repeat", C.c_int32), ("min_repeat_ms", C.c_double),
                ("max_number", C.c_int32), ("slow_cut", C.c_double), ("tol", C.c_double),
                ("check", C.c_int32), ("graph", C.c_int32)]


class ds_measurement(C.Structure):
    _fields_ = [("status", C.c_int32), ("n_repeats", C.c_int32), ("number", C.c_int32),
                ("cut", C.c_int32), ("median_ms", C.c_double), ("mean_ms", C.c_double),
                ("min_ms", C.c_double), ("first_ms", C.c_double), ("max_err", C.c_double),
                ("max_ref", C.c_double), ("nonfinite", C.c_int64),
                ("repeats_ms", C.c_double * DS_MAX_REPEATS)]

    def repeats(self):
        return [self.repeats_ms[i] for i in range(self.n_repeats)]


class ds_tune_io(C.Structure):
    _fields_ = [("x", C.c_void_p), ("w", C.c_void_p), ("y", C.c_void_p), ("ref", C.c_void_p),
                ("stream", C.c_void_p)]


class ds_tune_cfg(C.Structure):
    _fields_ = [("n_explore", C.c_int32), ("budget", C.c_int32), ("alpha", C.c_double),
                ("seed", C.c_uint64), ("frozen_mask", C.c_uint32), ("measure", ds_measure_cfg)]


class ds_tune_result(C.Structure):
    _fields_ = [("best", ds_sched), ("best_ms", C.c_double), ("seed_point", ds_sched),
                ("seed_ms", C.c_double), ("status", C.c_int32), ("n_explore_measured", C.c_int32),
                ("n_droplet_measured", C.c_int32), ("n_failed", C.c_int32), ("n_moves", C.c_int32),
                ("wall_s", C.c_double), ("explore_s", C.c_double), ("droplet_s", C.c_double),
                ("best_meas", ds_measurement)]


class ds_trace_entry(C.Structure):
    _fields_ = [("stage", C.c_int32), ("status", C.c_int32), ("key", C.c_uint64),
                ("median_ms", C.c_double)]


class ds_trace(C.Structure):
    _fields_ = [("entries", C.POINTER(ds_trace_entry)), ("cap", C.c_int32), ("n", C.c_int32)]


ds_measure_fn = C.CFUNCTYPE(C.c_int, C.c_void_p, C.POINTER(ds_sched), C.POINTER(ds_measurement))


class ds_exploit_cfg(C.Structure):
    _fields_ = [("kind", C.c_int32), ("budget", C.c_int32), ("seed", C.c_uint64),
                ("valid_only", C.c_int32), ("pop", C.c_int32), ("elite", C.c_int32),
                ("mutation", C.c_double)]


class ds_task(C.Structure):
    _fields_ = [("space", C.c_void_p), ("io", ds_tune_io), ("fn", ds_measure_fn),
                ("ctx", C.c_void_p), ("weight", C.c_double), ("seed", C.c_uint64)]


class ds_round(C.Structure):
    _fields_ = [("task", C.c_int32), ("trials", C.c_int32)]


DS_EXPLOIT_DROPLET, DS_EXPLOIT_RANDOM, DS_EXPLOIT_GRID, DS_EXPLOIT_GA = 0, 1, 2, 3
DS_EXPLOIT_DROPLET_LINE = 4

# name -> (restype, argtypes); the list is also the set of exported symbols
SIGNATURES = {
    "sched_space_create": (C.c_int, [C.c_int, C.POINTER(C.c_int64), C.c_int, C.POINTER(C.c_void_p)]),
    "sched_space_create_lattice": (C.c_int, [C.c_int, C.POINTER(C.c_int32), C.POINTER(C.c_int32),
                                             C.POINTER(C.c_uint64), C.c_int, C.POINTER(C.c_void_p)]),
    "sched_space_destroy": (None, [C.c_void_p]),
    "sched_space_info": (C.c_int, [C.c_void_p, C.POINTER(C.c_int), C.POINTER(C.c_int),
                                   C.POINTER(C.c_uint64)]),
    "sched_space_axis": (C.c_int, [C.c_void_p, C.c_int, C.POINTER(C.c_char_p), C.POINTER(C.c_int),
                                   C.POINTER(C.POINTER(C.c_int32))]),
    "sched_valid": (C.c_int, [C.c_void_p, C.POINTER(ds_sched)]),
    "sched_key": (C.c_int, [C.c_void_p, C.POINTER(ds_sched), C.POINTER(C.c_uint64)]),
    "sched_from_key": (C.c_int, [C.c_void_p, C.c_uint64, C.POINTER(ds_sched)]),
    "sched_neighbors": (C.c_int, [C.c_void_p, C.POINTER(ds_sched), C.POINTER(ds_sched), C.c_int,
                                  C.POINTER(C.c_int)]),
    "sched_origin": (C.c_int, [C.c_void_p, C.POINTER(ds_sched)]),
    "sched_geometry": (C.c_int, [C.c_void_p, C.POINTER(ds_sched), C.POINTER(ds_geometry)]),
    "ansor_draw": (C.c_int, [C.c_void_p, C.c_uint64, C.c_int, C.POINTER(ds_sched),
                             C.POINTER(C.c_int)]),
    "sched_has_kernel": (C.c_int, [C.c_void_p, C.POINTER(ds_sched)]),
    "sched_space_programs": (C.c_int, [C.c_void_p, C.POINTER(C.c_uint64), C.POINTER(C.c_int32),
                                       C.POINTER(C.c_uint64), C.c_int64, C.POINTER(C.c_int64)]),
    "sched_kernel_info": (C.c_int, [C.c_void_p, C.POINTER(ds_sched), C.c_int,
                                    C.POINTER(ds_kernel_info)]),
    "kernel_run": (C.c_int, [C.c_int, C.POINTER(ds_sched), C.c_void_p, C.c_void_p, C.c_void_p,
                             C.c_void_p]),
    "kernel_run_noalloc": (C.c_int, [C.c_int, C.POINTER(ds_sched), C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_void_p]),
    "kernel_run_reference": (C.c_int, [C.c_int, C.POINTER(C.c_int64), C.c_void_p, C.c_void_p,
                                       C.c_void_p, C.c_void_p]),
    "ds_measure_cfg_default": (None, [C.POINTER(ds_measure_cfg)]),
    "ds_measure": (C.c_int, [C.POINTER(ds_sched), C.POINTER(ds_tune_io), C.POINTER(ds_measure_cfg),
                             C.c_double, C.POINTER(ds_measurement)]),
    "ds_empty_kernel_floor": (C.c_int, [C.c_void_p, C.POINTER(ds_measure_cfg),
                                        C.POINTER(ds_measurement)]),
    "ds_mfma_ceiling": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int64, C.c_int,
                                  C.POINTER(ds_measure_cfg), C.POINTER(ds_measurement),
                                  C.POINTER(C.c_double)]),
    "ds_tune_cfg_default": (None, [C.POINTER(ds_tune_cfg)]),
    "ansor_sample": (C.c_int, [C.c_void_p, C.c_uint64, C.c_int, C.POINTER(ds_tune_io),
                               C.POINTER(ds_measure_cfg), C.POINTER(ds_sched),
                               C.POINTER(C.c_double), C.POINTER(ds_trace)]),
    "droplet_tune_ex": (C.c_int, [C.c_void_p, C.POINTER(ds_sched), C.c_int, C.POINTER(ds_tune_cfg),
                                  C.POINTER(ds_tune_io), ds_measure_fn, C.c_void_p,
                                  C.POINTER(ds_tune_result), C.POINTER(ds_trace)]),
    "ds_tune": (C.c_int, [C.c_void_p, C.POINTER(ds_tune_cfg), C.POINTER(ds_tune_io), ds_measure_fn,
                          C.c_void_p, C.POINTER(ds_tune_result), C.POINTER(ds_trace)]),
    "ds_cache_create": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p)]),
    "ds_cache_destroy": (None, [C.c_void_p]),
    "ds_cache_clone": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p)]),
    "ds_cache_size": (C.c_int, [C.c_void_p]),
    "ds_cache_get": (C.c_int, [C.c_void_p, C.POINTER(ds_sched), C.POINTER(ds_measurement)]),
    "ds_explore": (C.c_int, [C.c_void_p, C.POINTER(ds_tune_cfg), C.POINTER(ds_tune_io),
                             ds_measure_fn, C.c_void_p, C.c_void_p, C.POINTER(ds_tune_result),
                             C.POINTER(ds_trace)]),
    "ds_exploit_cfg_default": (None, [C.POINTER(ds_exploit_cfg)]),
    "ds_exploit": (C.c_int, [C.c_void_p, C.POINTER(ds_sched), C.POINTER(ds_exploit_cfg),
                             C.POINTER(ds_tune_cfg), C.POINTER(ds_tune_io), ds_measure_fn,
                             C.c_void_p, C.c_void_p, C.POINTER(ds_tune_result),
                             C.POINTER(ds_trace)]),
    "ds_tune_tasks": (C.c_int, [C.POINTER(ds_task), C.c_int, C.c_int, C.POINTER(ds_tune_cfg),
                                C.POINTER(ds_tune_result), C.POINTER(ds_round), C.c_int,
                                C.POINTER(C.c_int), C.POINTER(C.c_double)]),
    "droplet_tune": (C.c_int, [C.c_int, C.POINTER(C.c_int64), C.POINTER(ds_sched), C.c_int,
                               C.POINTER(ds_sched), C.POINTER(C.c_double)]),
    "ds_q8_quantize": (C.c_int, [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_void_p,
                                 C.c_void_p, C.c_void_p]),
    "ds_q8_matmul": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int64,
                               C.c_void_p]),
    "ds_swiglu8": (C.c_int, [C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64, C.c_int64,
                             C.c_void_p, C.c_void_p, C.c_void_p]),
    "ds_swiglu8_grad": (C.c_int, [C.c_void_p, C.c_void_p, C.c_int, C.c_int64, C.c_int64, C.c_int64,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]),
    "ds_rotary": (C.c_int, [C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_int, C.c_float, C.c_void_p,
                            C.c_void_p]),
    "ds_cache8_write": (C.c_int, [C.c_void_p] * 5),
    "ds_cache8_read": (C.c_int, [C.c_void_p] * 5),
    "ds_attn8": (C.c_int, [C.c_void_p] * 7 + [C.c_int64, C.c_void_p]),
    "ds_attn8_work": (C.c_int, [C.c_void_p] * 4 + [C.POINTER(C.c_int64)]),
    "ds_last_error": (C.c_char_p, []),
    "ds_gen_uniform": (C.c_int, [C.c_uint64, C.c_int64, C.POINTER(C.c_float)]),
    "ds_device_info": (C.c_int, [C.POINTER(C.c_int), C.POINTER(C.c_int), C.c_char_p, C.c_int]),
    "ds_num_instances": (C.c_int, []),
    "ds_shutdown": (None, []),
}

if not os.path.exists(LIB_PATH):
    raise RuntimeError(
        f"{LIB_PATH} is missing: build it with `python -m paper_2406_20037_amd.build` "
        "(there is no CPU fallback for the HIP path)")

lib = C.CDLL(LIB_PATH)
for _name, (_res, _args) in SIGNATURES.items():
    _f = getattr(lib, _name)
    _f.restype = _res
    _f.argtypes = _args


class DsError(RuntimeError):
    def __init__(self, func, rc):
        msg = lib.ds_last_error()
        super().__init__(f"{func} -> {STATUS_NAMES.get(rc, rc)}: {msg.decode() if msg else ''}")
        self.rc = rc


def check(func, rc):
    if rc < 0:
        raise DsError(func, rc)
    return rc


def ptr(t):
    """Device address of a tensor or an integer address."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return int(t.data_ptr())


def stream_handle(stream=None):
    if stream is None:
        try:
            import torch
            if torch.cuda.is_available():
                return int(torch.cuda.current_stream().cuda_stream) or None
        except Exception:
            pass
        return None
    if isinstance(stream, int):
        return stream or None
    return int(stream.cuda_stream) or None


def make_io(x, w, y, ref=None, stream=None):
    return ds_tune_io(ptr(x), ptr(w), ptr(y), ptr(ref), stream_handle(stream))


def measure_cfg(**kw):
    cfg = ds_measure_cfg()
    lib.ds_measure_cfg_default(C.byref(cfg))
    for k, v in kw.items():
        setattr(cfg, k, v)
    return cfg


def tune_cfg(measure=None, **kw):
    cfg = ds_tune_cfg()
    lib.ds_tune_cfg_default(C.byref(cfg))
    for k, v in kw.items():
        setattr(cfg, k, v)
    if measure is not None:
        cfg.measure = measure
    return cfg


class Space:
    """A ``ds_space`` handle (sched_space_create / sched_space_create_lattice)."""

    def __init__(self, op=None, shape=None, *, lattice=None, invalid_keys=()):
        h = C.c_void_p()
        if lattice is not None:
            nv = (C.c_int32 * len(lattice))(*[len(v) for v in lattice])
            flat = [int(x) for v in lattice for x in v]
            vals = (C.c_int32 * len(flat))(*flat)
            inv = (C.c_uint64 * max(1, len(invalid_keys)))(*invalid_keys)
            check("sched_space_create_lattice",
                  lib.sched_space_create_lattice(len(lattice), nv, vals, inv, len(invalid_keys),
                                                 C.byref(h)))
        else:
            sh = (C.c_int64 * len(shape))(*[int(v) for v in shape])
            check("sched_space_create", lib.sched_space_create(op, sh, len(shape), C.byref(h)))
        self.h = h
        op_, nk, size = C.c_int(), C.c_int(), C.c_uint64()
        check("sched_space_info", lib.sched_space_info(h, C.byref(op_), C.byref(nk), C.byref(size)))
        self.op, self.nknobs, self.size = op_.value, nk.value, size.value
        self.shape = tuple(int(v) for v in shape) if shape is not None else ()
        self.names, self.values = [], []
        for a in range(self.nknobs):
            name, n, vals = C.c_char_p(), C.c_int(), C.POINTER(C.c_int32)()
            check("sched_space_axis",
                  lib.sched_space_axis(h, a, C.byref(name), C.byref(n), C.byref(vals)))
            self.names.append(name.value.decode())
            self.values.append([vals[i] for i in range(n.value)])
        self.sizes = [len(v) for v in self.values]

    def __del__(self):
        h = getattr(self, "h", None)
        if h and lib is not None:
            try:
                lib.sched_space_destroy(h)
            except Exception:   # interpreter shutdown
                pass
            self.h = None

    def sched(self, idx):
        s = ds_sched()
        s.op = self.op
        s.nknobs = self.nknobs
        for i, v in enumerate(self.shape):
            s.shape[i] = v
        for a, i in enumerate(idx):
            s.idx[a] = int(i)
        return s

    def sched_of(self, **knobs):
        return self.sched([self.values[a].index(knobs[n]) for a, n in enumerate(self.names)])

    def knobs(self, s):
        idx = s.index() if isinstance(s, ds_sched) else tuple(s)
        return {n: self.values[a][i] for a, (n, i) in enumerate(zip(self.names, idx))}

    def valid(self, idx):
        return bool(check("sched_valid", lib.sched_valid(self.h, C.byref(self.sched(idx)))))

    def key(self, idx):
        k = C.c_uint64()
        check("sched_key", lib.sched_key(self.h, C.byref(self.sched(idx)), C.byref(k)))
        return k.value

    def from_key(self, key):
        s = ds_sched()
        check("sched_from_key", lib.sched_from_key(self.h, key, C.byref(s)))
        return s.index()

    def neighbors(self, idx):
        out = (ds_sched * (2 * DS_MAX_KNOBS))()
        n = C.c_int()
        check("sched_neighbors",
              lib.sched_neighbors(self.h, C.byref(self.sched(idx)), out, len(out), C.byref(n)))
        return [out[i].index() for i in range(n.value)]

    def origin(self):
        s = ds_sched()
        check("sched_origin", lib.sched_origin(self.h, C.byref(s)))
        return s.index()

    def geometry(self, idx):
        g = ds_geometry()
        check("sched_geometry", lib.sched_geometry(self.h, C.byref(self.sched(idx)), C.byref(g)))
        return dict(valid=bool(g.valid), grid=g.grid, threads=g.threads, lds_bytes=g.lds_bytes,
                    acc=g.acc, unroll_eff=g.unroll_eff, t0=g.t0, t1=g.t1, red=g.red,
                    chunks=g.chunks)

    def has_kernel(self, idx):
        return bool(check("sched_has_kernel", lib.sched_has_kernel(self.h, C.byref(self.sched(idx)))))

    def kernel_info(self, idx, with_attrs=False):
        """Compiled instance, launch geometry and argument hash of a valid point."""
        out = ds_kernel_info()
        check("sched_kernel_info", lib.sched_kernel_info(self.h, C.byref(self.sched(idx)),
                                                         int(with_attrs), C.byref(out)))
        return out.as_dict()

    def programs(self):
        """(keys, instances, args_hashes) of every valid point, key order (numpy)."""
        import numpy as np
        n = C.c_int64()
        check("sched_space_programs", lib.sched_space_programs(self.h, None, None, None, 0,
                                                               C.byref(n)))
        keys = np.zeros(max(1, n.value), np.uint64)
        inst = np.zeros(max(1, n.value), np.int32)
        hashes = np.zeros(max(1, n.value), np.uint64)
        check("sched_space_programs", lib.sched_space_programs(
            self.h, keys.ctypes.data_as(C.POINTER(C.c_uint64)),
            inst.ctypes.data_as(C.POINTER(C.c_int32)),
            hashes.ctypes.data_as(C.POINTER(C.c_uint64)), n.value, C.byref(n)))
        return keys[: n.value], inst[: n.value], hashes[: n.value]

    def draw(self, seed, n):
        out = (ds_sched * max(1, n))()
        m = C.c_int()
        rc = lib.ansor_draw(self.h, C.c_uint64(seed), n, out, C.byref(m))
        if rc != DS_EEXHAUSTED:
            check("ansor_draw", rc)
        return [out[i].index() for i in range(m.value)]


def kernel_run(op, sched, x, w, y, stream=None):
    return check("kernel_run", lib.kernel_run(op, C.byref(sched), ptr(x), ptr(w), ptr(y),
                                              stream_handle(stream)))


def kernel_run_noalloc(op, sched, x, w, y, stream=None):
    return check("kernel_run_noalloc",
                 lib.kernel_run_noalloc(op, C.byref(sched), ptr(x), ptr(w), ptr(y),
                                        stream_handle(stream)))


def kernel_run_reference(op, shape, x, w, y, stream=None):
    sh = (C.c_int64 * len(shape))(*[int(v) for v in shape])
    return check("kernel_run_reference",
                 lib.kernel_run_reference(op, sh, ptr(x), ptr(w), ptr(y), stream_handle(stream)))


def ds_measure(sched, io, cfg=None, best_so_far_ms=0.0):
    m = ds_measurement()
    check("ds_measure", lib.ds_measure(C.byref(sched), C.byref(io),
                                       C.byref(cfg) if cfg is not None else None,
                                       best_so_far_ms, C.byref(m)))
    return m


def ds_empty_kernel_floor(stream=None, cfg=None):
    m = ds_measurement()
    check("ds_empty_kernel_floor",
          lib.ds_empty_kernel_floor(stream_handle(stream), C.byref(cfg) if cfg else None,
                                    C.byref(m)))
    return m


DS_MFMA_CEILING_SINK = 262144


def ds_mfma_ceiling(sink, iters=512, stream=None, cfg=None):
    """(measurement, flop per launch) of the library's pure-MFMA calibration
    kernel; sink is a float32 device tensor of >= DS_MFMA_CEILING_SINK elements."""
    m = ds_measurement()
    flop = C.c_double()
    check("ds_mfma_ceiling",
          lib.ds_mfma_ceiling(stream_handle(stream), ptr(sink), sink.numel(), iters,
                              C.byref(cfg) if cfg else None, C.byref(m), C.byref(flop)))
    return m, flop.value


def _trace(cap):
    if not cap:
        return None, None
    arr = (ds_trace_entry * cap)()
    return arr, ds_trace(C.cast(arr, C.POINTER(ds_trace_entry)), cap, 0)


def _trace_list(arr, tr):
    if tr is None:
        return None
    return [(arr[i].stage, arr[i].status, arr[i].key, arr[i].median_ms)
            for i in range(min(tr.n, tr.cap))]


def _callback(fn):
    """Wraps fn(idx) -> float | list[float] | None (failure) as a ds_measure_fn."""
    if fn is None:
        return ds_measure_fn(), None

    def cb(ctx, s, out):
        try:
            v = fn(s.contents.index())
        except Exception:
            return DS_EHIP
        if v is None:
            return DS_EHIP
        reps = list(v) if isinstance(v, (list, tuple)) else [float(v)]
        m = out.contents
        m.status = 0
        m.n_repeats = min(len(reps), DS_MAX_REPEATS)
        for i in range(m.n_repeats):
            m.repeats_ms[i] = reps[i]
        srt = sorted(reps)
        n = len(srt)
        m.median_ms = srt[n // 2] if n % 2 else 0.5 * (srt[n // 2 - 1] + srt[n // 2])
        return DS_OK

    c = ds_measure_fn(cb)
    return c, c


def ansor_sample(space, seed, n_explore, io, cfg=None, trace_cap=0):
    best, ms = ds_sched(), C.c_double()
    arr, tr = _trace(trace_cap)
    check("ansor_sample", lib.ansor_sample(space.h, C.c_uint64(seed), n_explore, C.byref(io),
                                           C.byref(cfg) if cfg else None, C.byref(best),
                                           C.byref(ms), C.byref(tr) if tr else None))
    return best, ms.value, _trace_list(arr, tr)


def droplet_tune_ex(space, start, budget, cfg=None, io=None, cost=None, trace_cap=0):
    res = ds_tune_result()
    arr, tr = _trace(trace_cap)
    cb, keep = _callback(cost)
    st = space.sched(start) if start is not None and not isinstance(start, ds_sched) else start
    check("droplet_tune_ex",
          lib.droplet_tune_ex(space.h, C.byref(st) if st is not None else None, budget,
                              C.byref(cfg) if cfg else None, C.byref(io) if io else None, cb, None,
                              C.byref(res), C.byref(tr) if tr else None))
    del keep
    return res, _trace_list(arr, tr)


def ds_tune(space, cfg=None, io=None, cost=None, trace_cap=0):
    res = ds_tune_result()
    arr, tr = _trace(trace_cap)
    cb, keep = _callback(cost)
    check("ds_tune", lib.ds_tune(space.h, C.byref(cfg) if cfg else None,
                                 C.byref(io) if io else None, cb, None, C.byref(res),
                                 C.byref(tr) if tr else None))
    del keep
    return res, _trace_list(arr, tr)


def exploit_cfg(**kw):
    cfg = ds_exploit_cfg()
    lib.ds_exploit_cfg_default(C.byref(cfg))
    for k, v in kw.items():
        setattr(cfg, k, v)
    return cfg


class Cache:
    """Owns a ds_cache of one space."""

    def __init__(self, space, _handle=None):
        self.space = space
        self.h = C.c_void_p(_handle) if _handle else C.c_void_p()
        if not _handle:
            check("ds_cache_create", lib.ds_cache_create(space.h, C.byref(self.h)))

    def __del__(self):
        try:
            if self.h:
                lib.ds_cache_destroy(self.h)
                self.h = C.c_void_p()
        except Exception:
            pass

    def clone(self):
        h = C.c_void_p()
        check("ds_cache_clone", lib.ds_cache_clone(self.h, C.byref(h)))
        return Cache(self.space, h.value)

    def __len__(self):
        n = lib.ds_cache_size(self.h)
        check("ds_cache_size", min(n, 0))
        return n

    def get(self, idx):
        """The cached ds_measurement of idx, or None."""
        m = ds_measurement()
        s = self.space.sched(idx) if not isinstance(idx, ds_sched) else idx
        rc = lib.ds_cache_get(self.h, C.byref(s), C.byref(m))
        check("ds_cache_get", min(rc, 0))
        return m if rc == 1 else None


def ds_explore(space, cache, cfg=None, io=None, cost=None, trace_cap=0):
    res = ds_tune_result()
    arr, tr = _trace(trace_cap)
    cb, keep = _callback(cost)
    check("ds_explore", lib.ds_explore(space.h, C.byref(cfg) if cfg else None,
                                       C.byref(io) if io else None, cb, None, cache.h,
                                       C.byref(res), C.byref(tr) if tr else None))
    del keep
    return res, _trace_list(arr, tr)


def ds_exploit(space, start, ecfg=None, cfg=None, io=None, cost=None, cache=None, trace_cap=0):
    res = ds_tune_result()
    arr, tr = _trace(trace_cap)
    cb, keep = _callback(cost)
    st = start if isinstance(start, ds_sched) else space.sched(start)
    check("ds_exploit", lib.ds_exploit(space.h, C.byref(st), C.byref(ecfg) if ecfg else None,
                                       C.byref(cfg) if cfg else None, C.byref(io) if io else None,
                                       cb, None, cache.h if cache is not None else None,
                                       C.byref(res), C.byref(tr) if tr else None))
    del keep
    return res, _trace_list(arr, tr)


def ds_tune_tasks(spaces, weights, seeds, total_trials, cfg=None, ios=None, costs=None,
                  rounds_cap=4096):
    """One exploration budget over several tasks, then Droplet per task.
    Returns (results[list of ds_tune_result], rounds[list of (task, n)], network_ms)."""
    n = len(spaces)
    tasks = (ds_task * n)()
    keep = []
    for t in range(n):
        tasks[t].space = spaces[t].h
        if ios is not None:
            tasks[t].io = ios[t]
        cb, k = _callback(costs[t] if costs is not None else None)
        keep.append(k)
        tasks[t].fn = cb
        tasks[t].weight = float(weights[t])
        tasks[t].seed = int(seeds[t])
    results = (ds_tune_result * n)()
    rounds = (ds_round * max(1, rounds_cap))()
    nr, net = C.c_int(), C.c_double()
    check("ds_tune_tasks", lib.ds_tune_tasks(tasks, n, int(total_trials),
                                             C.byref(cfg) if cfg else None, results, rounds,
                                             rounds_cap, C.byref(nr), C.byref(net)))
    del keep
    return (list(results), [(rounds[i].task, rounds[i].trials) for i in range(min(nr.value, rounds_cap))],
            net.value)


def droplet_tune(op, shape, start=None, budget=100):
    sh = (C.c_int64 * len(shape))(*[int(v) for v in shape])
    best, ms = ds_sched(), C.c_double()
    check("droplet_tune", lib.droplet_tune(op, sh, C.byref(start) if start is not None else None,
                                           budget, C.byref(best), C.byref(ms)))
    return best, ms.value


class Q8:
    """An 8-bit matrix with a scale for each block of 128 along a row (or, with
    ``block_rows=128``, each 128x128 square): ``data`` [rows, cols] of
    ``torch.float8_e4m3fn`` or ``float8_e5m2`` and ``scale`` [ceil(rows / block_rows),
    ceil(cols / 128)] of ``torch.float8_e8m0fnu`` (powers of two) or ``float32``.
    Q8(rows, cols) allocates both, uninitialised; Q8.of wraps tensors that exist.

    The operators below run on the one GPU that holds their operands, on its current
    stream unless one is given, and raise ValueError for operands in host memory or on
    several GPUs."""

    def __init__(self, rows, cols, dtype=None, *, scale=None, block_rows=1, device="cuda"):
        dtype = dtype or _torch.float8_e4m3fn
        scale = scale or _torch.float8_e8m0fnu
        ld = max(16, (cols + 15) // 16 * 16)
        data = _torch.empty(rows, ld, dtype=_torch.uint8, device=device).view(dtype)[:, :cols]
        nr, nc = -(-rows // block_rows), -(-cols // DS_Q8_BLOCK)
        # rows of scales in whole 4-byte words: products copy them so
        sc = _torch.empty(nr, (nc + 3) // 4 * 4, dtype=scale, device=device)[:, :nc]
        self._wrap(data, sc, block_rows)

    @classmethod
    def of(cls, data, scale, block_rows=1):
        """The matrix held in data and scale, which it shares: rows of data a multiple
        of 16 bytes apart, elements of a row side by side."""
        m = cls.__new__(cls)
        m._wrap(data, scale, block_rows)
        return m

    def _wrap(self, data, scale, block_rows):
        fmt = {_torch.float8_e4m3fn: DS_Q8_E4M3, _torch.float8_e5m2: DS_Q8_E5M2}.get(data.dtype)
        kind = {_torch.float8_e8m0fnu: DS_SCALE_POW2, _torch.float32: DS_SCALE_F32}.get(scale.dtype)
        if fmt is None or kind is None:
            raise TypeError(f"8-bit values of {data.dtype} with scales of {scale.dtype}")
        if block_rows not in (1, DS_Q8_BLOCK):
            raise ValueError(f"block_rows is 1 or {DS_Q8_BLOCK}, not {block_rows}")
        rows, cols, ld = _plain_rows(data)
        want = (-(-rows // block_rows), -(-cols // DS_Q8_BLOCK))
        if tuple(scale.shape) != want:
            raise ValueError(f"scales of shape {tuple(scale.shape)}, not {want}")
        if scale.device != data.device:
            raise ValueError(f"values on {data.device}, scales on {scale.device}")
        sld = _plain_rows(scale)[2]
        if rows <= 1:                   # the stride of a single row says nothing
            ld = max(16, (cols + 15) // 16 * 16)
        if want[0] <= 1:                # (in whole words where it allows them: products copy scales so)
            sld = min(sld, (want[1] + 3) // 4 * 4)
        self.data, self.scale, self.rows, self.cols = data, scale, rows, cols
        self.block_rows = block_rows
        self._device = data.get_device()
        self._c = ds_q8(data.data_ptr(), scale.data_ptr(), rows, cols, ld, sld, fmt, kind, block_rows, 0)
        self._p = C.addressof(self._c)

    def values(self):
        """The fp32 values that it stands for (a new tensor)."""
        s = self.scale.to(_torch.float32)
        if self.block_rows != 1:
            s = s.repeat_interleave(self.block_rows, 0)[: self.rows]
        return self.data.to(_torch.float32) * s.repeat_interleave(DS_Q8_BLOCK, 1)[:, : self.cols]


_PLAIN = {} if _torch is None else {_torch.float32: DS_TYPE_F32, _torch.float16: DS_TYPE_F16,
                                    _torch.bfloat16: DS_TYPE_BF16}


def _plain_rows(t):
    """(rows, cols, elements between rows) of a 2-D tensor whose rows' elements are side by side."""
    rows, cols = t.shape
    ld, one = t.stride()
    if one != 1 and cols > 1:
        raise ValueError(f"elements of a row are {one} apart, not side by side")
    return rows, cols, ld if rows > 1 else max(ld, cols)


def _plain(t):
    if t.dtype not in _PLAIN:
        raise TypeError(f"fp32, fp16 or bf16, not {t.dtype}")
    return (t.data_ptr(), _PLAIN[t.dtype], *_plain_rows(t))


def _q8_device(first, *rest):
    """The one GPU of operands with these device indices (-1: host memory, None: no operand)."""
    one = first >= 0
    for d in rest:
        one = one and (d is None or d == first)
    if not one:
        raise ValueError("operands on " + ", ".join("the host" if d < 0 else f"GPU {d}" for d in (first, *rest)
                                                    if d is not None) + ", not on one GPU")
    return first


# the current stream's handle without a Stream object (2.5 us of a call's 7)
_raw_stream = getattr(getattr(_torch, "_C", None), "_cuda_getCurrentRawStream", None)


def _q8_stream(stream, dev):
    if stream is not None:
        if getattr(stream, "device_index", dev) != dev:
            raise ValueError(f"a stream of GPU {stream.device_index}, operands on GPU {dev}")
        return stream_handle(stream)
    if _raw_stream is not None:
        return _raw_stream(dev)
    return _torch.cuda.current_stream(dev).cuda_stream


def ds_q8_quantize(x, row=None, col=None, stream=None):
    """x [rows, cols] (fp32, fp16, bf16) in 8 bits: in row (a Q8 of x's shape), transposed in
    col (a Q8 of cols x rows), or both."""
    p, t, rows, cols, ld = _plain(x)
    dev = _q8_device(x.get_device(), row and row._device, col and col._device)
    if dev != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return ds_q8_quantize(x, row, col, stream)
    return check("ds_q8_quantize", lib.ds_q8_quantize(p, t, rows, cols, ld, row and row._p,
                                                      col and col._p, _q8_stream(stream, dev)))


def ds_q8_matmul(a, b, c, stream=None, exact=False):
    """c = a b^T of two Q8; c fp32, fp16 or bf16.  exact: sums exact to fp32 for a 16-bit c of any
    size, as an fp32 c and one of few rows always have them."""
    p, t, rows, cols, ld = _plain(c)
    if rows != a.rows or cols != b.rows:
        raise ValueError(f"c is {rows} x {cols}, not {a.rows} x {b.rows}")
    dev = _q8_device(c.get_device(), a._device, b._device)
    if dev != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return ds_q8_matmul(a, b, c, stream, exact)
    if exact:
        t += DS_EXACT_SUMS
    return check("ds_q8_matmul", lib.ds_q8_matmul(a._p, b._p, p, t, ld, _q8_stream(stream, dev)))


def ds_swiglu8(gu, h, saved=None, stream=None):
    """silu(gate) * other of gu [rows, up + hidden] in the Q8 h [rows, hidden]; gu itself, the
    checkpoint of the backward pass, in the Q8 saved unless that is None."""
    p, t, rows, cols, ld = _plain(gu)
    if rows != h.rows:
        raise ValueError(f"gu has {rows} rows, h {h.rows}")
    dev = _q8_device(gu.get_device(), h._device, saved and saved._device)
    if dev != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return ds_swiglu8(gu, h, saved, stream)
    return check("ds_swiglu8", lib.ds_swiglu8(p, t, rows, h.cols, cols - h.cols, ld, h._p,
                                              saved and saved._p, _q8_stream(stream, dev)))


def ds_swiglu8_grad(saved, dh, dgu=None, dgu_t=None, h_t=None, stream=None):
    """The gradient of gu from the checkpoint and dh [rows, hidden], in dgu and transposed in
    dgu_t, and the unit's output transposed in h_t (each a Q8 or None)."""
    p, t, rows, cols, ld = _plain(dh)
    if rows != saved.rows:
        raise ValueError(f"dh has {rows} rows, saved {saved.rows}")
    dev = _q8_device(dh.get_device(), saved._device, dgu and dgu._device, dgu_t and dgu_t._device,
                     h_t and h_t._device)
    if dev != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return ds_swiglu8_grad(saved, dh, dgu, dgu_t, h_t, stream)
    return check("ds_swiglu8_grad",
                 lib.ds_swiglu8_grad(saved._p, p, t, cols, saved.cols - cols, ld, dgu and dgu._p,
                                     dgu_t and dgu_t._p, h_t and h_t._p, _q8_stream(stream, dev)))


class Cache8:
    """Keys and values of sequences in 8 bits, in pages of ``page`` tokens: ``k`` and ``v`` [pages, heads,
    page, dim] of ``torch.float8_e4m3fn`` or ``float8_e5m2``, and one scale a row in ``k_scale`` and
    ``v_scale`` [pages, heads, page] of ``torch.float8_e8m0fnu`` (powers of two) or ``float32``.
    Cache8(pages, heads, dim) allocates them, uninitialised: what no token was written to is never
    used.  Cache8.of wraps tensors that exist.

    The operators on it run as those of Q8 do: on the one GPU that holds their operands, on its current
    stream unless one is given."""

    def __init__(self, pages, heads, dim, page=64, dtype=None, *, scale=None, device="cuda"):
        def rows():
            return _torch.empty(pages, heads, page, dim, dtype=_torch.uint8,
                                device=device).view(dtype or _torch.float8_e4m3fn)

        def scales():
            return _torch.empty(pages, heads, page, dtype=scale or _torch.float8_e8m0fnu, device=device)
        self._wrap(rows(), rows(), scales(), scales())

    @classmethod
    def of(cls, k, v, k_scale, v_scale):
        """The cache held in these tensors, which it shares.  Pages may lie apart (k and v the halves of one
        tensor), as far in k as in v; what is inside a page lies in order."""
        c = cls.__new__(cls)
        c._wrap(k, v, k_scale, v_scale)
        return c

    def _wrap(self, k, v, k_scale, v_scale):
        fmt = {_torch.float8_e4m3fn: DS_Q8_E4M3, _torch.float8_e5m2: DS_Q8_E5M2}.get(k.dtype)
        kind = {_torch.float8_e8m0fnu: DS_SCALE_POW2, _torch.float32: DS_SCALE_F32}.get(k_scale.dtype)
        if fmt is None or kind is None or v.dtype != k.dtype or v_scale.dtype != k_scale.dtype:
            raise TypeError(f"a cache of {k.dtype} and {v.dtype} with scales of {k_scale.dtype} and {v_scale.dtype}")
        pages, heads, page, dim = k.shape
        if v.shape != k.shape or tuple(k_scale.shape) != (pages, heads, page) or v_scale.shape != k_scale.shape:
            raise ValueError(f"k {tuple(k.shape)}, v {tuple(v.shape)}, scales {tuple(k_scale.shape)} and "
                             f"{tuple(v_scale.shape)}")
        if len({t.get_device() for t in (k, v, k_scale, v_scale)}) != 1:
            raise ValueError("k, v and their scales are not on one device")
        stride = [_page_stride(t) for t in (k, v)]
        sstride = [_page_stride(t) for t in (k_scale, v_scale)]
        if pages > 1 and (stride[0] != stride[1] or sstride[0] != sstride[1]):
            raise ValueError(f"pages {stride} bytes and {sstride} scales apart")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.pages, self.heads, self.page, self.dim = pages, heads, page, dim
        self._device = k.get_device()
        self._c = ds_cache8(k.data_ptr(), v.data_ptr(), k_scale.data_ptr(), v_scale.data_ptr(), pages, stride[0],
                            sstride[0], page, heads, dim, fmt, kind, 0)
        self._p = C.addressof(self._c)

    def values(self):
        """The fp32 values of all pages' keys and values (new tensors)."""
        return tuple(x.to(_torch.float32) * s.to(_torch.float32)[..., None]
                     for x, s in ((self.k, self.k_scale), (self.v, self.v_scale)))


def _page_stride(t):
    """Elements between pages of a cache's tensor whose pages are whole."""
    want = 1
    for n, s in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if n > 1 and s != want:
            raise ValueError(f"a page's elements do not lie in order: strides {t.stride()} of {tuple(t.shape)}")
        want *= n
    return t.stride(0) if t.shape[0] > 1 else (want + 15) // 16 * 16


class Chunk:
    """What a call's new tokens belong to: int32 tensors on the GPU, whose contents may change between calls
    and replays.  Sequence b has tokens starts[b] .. starts[b + 1] - 1 (``starts`` [seqs + 1]), the last of
    its ``lengths[b]`` tokens; its token at position p lies in page ``table[b, p // page]``."""

    def __init__(self, starts, lengths, table):
        for name, t, dims in (("starts", starts, 1), ("lengths", lengths, 1), ("table", table, 2)):
            if t.dtype != _torch.int32 or t.dim() != dims:
                raise TypeError(f"{name}: {t.dtype} of {t.dim()} dimensions, not int32 of {dims}")
            if t.shape[-1] > 1 and t.stride(-1) != 1:
                raise ValueError(f"{name}: elements {t.stride(-1)} apart, not side by side")
        seqs = lengths.shape[0]
        if starts.shape[0] != seqs + 1 or table.shape[0] != seqs:
            raise ValueError(f"{starts.shape[0]} starts and {table.shape[0]} rows of pages of {seqs} sequences")
        if not starts.get_device() == lengths.get_device() == table.get_device():
            raise ValueError("starts, lengths and table are not on one device")
        self.starts, self.lengths, self.table = starts, lengths, table
        self._device = starts.get_device()
        cols = table.shape[1]
        ld = table.stride(0) if seqs > 1 else max(cols, table.stride(0))
        self._c = ds_chunk(starts.data_ptr(), lengths.data_ptr(), table.data_ptr(), seqs, cols, ld)
        self._p = C.addressof(self._c)


# the bytes of a ds_heads and of a ds_attn8_cfg (a third of the time of the ctypes structure)
_pack_heads = struct.Struct("@Pqqqqqii").pack
_pack_cfg = struct.Struct("@diiqq").pack


def _heads(t, more=0):
    """The C form of a tensor [tokens, heads, dim] whose rows' elements are side by side; more: added to its type."""
    kind = _PLAIN.get(t.dtype)
    if kind is None:
        raise TypeError(f"fp32, fp16 or bf16, not {t.dtype}")
    tokens, heads, dim = t.shape
    ld, hld, one = t.stride()
    if one != 1 and dim > 1:
        raise ValueError(f"elements of a row are {one} apart, not side by side")
    return _pack_heads(t.data_ptr(), tokens, heads, dim, ld, hld, kind + more, 0)


def _list(t, dtype, n, what):
    if t.dtype != dtype or t.dim() != 1 or t.shape[0] != n or (n > 1 and t.stride(0) != 1):
        raise ValueError(f"{what}: {t.dtype} of shape {tuple(t.shape)}, not {n} of {dtype} side by side")
    return t.data_ptr()


def ds_rotary(x, pos, freqs, y=None, *, pairs=False, scale=1.0, inverse=False, stream=None):
    """x [tokens, heads, dim] turned by its tokens' positions (pos [tokens], int32) in y, or in place:
    pair i of the first 2 * len(freqs) values of each head by pos * freqs[i] (fp32), times scale.
    pairs: values 2 i and 2 i + 1 in place of i and i + len(freqs).  inverse: by the opposite angle, which
    takes the gradient of y to the gradient of x."""
    y = x if y is None else y
    dev = _q8_device(x.get_device(), pos.get_device(), freqs.get_device(), y.get_device())
    if dev != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return ds_rotary(x, pos, freqs, y, pairs=pairs, scale=scale, inverse=inverse, stream=stream)
    mode = (DS_ROTARY_PAIRS if pairs else DS_ROTARY_HALVES) + (DS_ROTARY_INVERSE if inverse else 0)
    n = freqs.numel()
    hx = _heads(x)
    return check("ds_rotary", lib.ds_rotary(hx, _list(pos, _torch.int32, x.shape[0], "pos"),
                                            _list(freqs, _torch.float32, n, "freqs"), 2 * n, mode, scale,
                                            hx if y is x else _heads(y), _q8_stream(stream, dev)))


def _cache8_rows(name, cache, chunk, k, v, stream):
    dev = _q8_device(cache._device, chunk._device, k.get_device(), v.get_device())
    if dev != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return _cache8_rows(name, cache, chunk, k, v, stream)
    return check(name, getattr(lib, name)(cache._p, chunk._p, _heads(k), _heads(v), _q8_stream(stream, dev)))


def ds_cache8_write(cache, chunk, k, v, stream=None):
    """The rows of k and v [tokens, cache heads, dim] (fp32, fp16, bf16) in 8 bits to the places of their
    tokens in the cache."""
    return _cache8_rows("ds_cache8_write", cache, chunk, k, v, stream)


def ds_cache8_read(cache, chunk, k, v, stream=None):
    """The rows of the tokens' places in the cache back in k and v [tokens, cache heads, dim]."""
    return _cache8_rows("ds_cache8_read", cache, chunk, k, v, stream)


def ds_attn8_work(q, cache, chunk, *, scale=None, causal=True, window=0, max_len=0, exact=False):
    """Bytes of the workspace of ds_attn8 with these arguments."""
    n = C.c_int64()
    cfg = _pack_cfg(q.shape[2] ** -0.5 if scale is None else scale, causal, 0, window, max_len)
    check("ds_attn8_work", lib.ds_attn8_work(_heads(q, DS_EXACT_SUMS if exact else 0), cache._p, chunk._p, cfg, C.byref(n)))
    return n.value


def ds_attn8(q, cache, chunk, out, lse=None, *, scale=None, causal=True, window=0, max_len=0, work=None,
             stream=None, exact=False):
    """Attention of q [tokens, heads, dim] over the keys and values of the tokens' sequences in the cache, in
    out; log of the sums in lse [tokens, heads] (fp32) unless that is None.  scale: dim ** -0.5 unless given.
    causal: keys up to the token's own position, the latest ``window`` of them if that is not 0.  max_len: no sequence
    is longer (0: what the table holds); a low one keeps the split of few tokens' work even.
    work: a uint8 tensor of ds_attn8_work bytes, this call's until it is done; allocated if None.
    exact: weights in two parts for bf16 q over powers of two, as all other types have them."""
    dev = _q8_device(q.get_device(), cache._device, chunk._device, out.get_device(), lse if lse is None else lse.get_device(),
                     work if work is None else work.get_device())
    if dev != _torch.cuda.current_device():
        with _torch.cuda.device(dev):
            return ds_attn8(q, cache, chunk, out, lse, scale=scale, causal=causal, window=window, max_len=max_len,
                            work=work, stream=stream, exact=exact)
    cfg = _pack_cfg(q.shape[2] ** -0.5 if scale is None else scale, causal, 0, window, max_len)
    qh, oh = _heads(q, DS_EXACT_SUMS if exact else 0), _heads(out)
    if lse is not None and (lse.dtype != _torch.float32 or tuple(lse.shape) != tuple(q.shape[:2]) or
                            not lse.is_contiguous()):
        raise ValueError(f"lse: {lse.dtype} of shape {tuple(lse.shape)}, not float32 of {tuple(q.shape[:2])}")
    handle = _q8_stream(stream, dev)
    if work is None:
        n = C.c_int64()
        check("ds_attn8", lib.ds_attn8_work(qh, cache._p, chunk._p, cfg, C.byref(n)))
        need = n.value
        if need:
            if stream is None:
                work = _torch.empty(need, dtype=_torch.uint8, device=q.device)
            else:                        # the stream's own memory: it is given back in its order
                with _torch.cuda.stream(_torch.cuda.ExternalStream(handle or 0, device=q.device)
                                        if isinstance(stream, int) else stream):
                    work = _torch.empty(need, dtype=_torch.uint8, device=q.device)
    else:
        if work.dtype != _torch.uint8 or not work.is_contiguous():
            raise ValueError(f"work: {work.dtype}, not uint8 side by side")
        need = work.numel()
    return check("ds_attn8", lib.ds_attn8(qh, cache._p, chunk._p, cfg, oh, ptr(lse), ptr(work), need, handle))


def ds_gen_uniform(seed, n):
    buf = (C.c_float * max(1, n))()
    check("ds_gen_uniform", lib.ds_gen_uniform(C.c_uint64(seed), n, buf))
    return buf


def ds_device_info():
    cus, clk = C.c_int(), C.c_int()
    arch = C.create_string_buffer(64)
    check("ds_device_info", lib.ds_device_info(C.byref(cus), C.byref(clk), arch, 64))
    return dict(cus=cus.value, clock_khz=clk.value, arch=arch.value.decode())


def ds_num_instances():
    return lib.ds_num_instances()


def ds_shutdown():
    lib.ds_shutdown()
