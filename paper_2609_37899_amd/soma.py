"""Thin Python binding of ``libsoma.so`` (include/soma.h): argument marshalling only.

Every step of the SPSA hot path runs in the HIP library.  torch supplies
device memory and the stream; nothing here computes.  If the library is not
built (``python -m paper_2609_37899_amd.build``), every call raises.
"""
from __future__ import annotations

import ctypes
import os
from dataclasses import dataclass

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libsoma.so")

SOMA_OK, SOMA_EINVAL, SOMA_ESHAPE, SOMA_EDEVICE, SOMA_EWORKSPACE = 0, -1, -2, -3, -4
LOSS_INDEPENDENT, LOSS_SUMMED = 0, 1
PROBE_GAUSSIAN, PROBE_SPARSE_RADEMACHER, PROBE_RADEMACHER = 0, 1, 2
FLAG_PER_STEP_RECURRENCE = 1
FLAG_TILED_WEIGHTS = 2
FLAG_STAGED_RECURRENCE = 4
FLAG_FP32_SEQUENCE = 8
ARCH_LSTM, ARCH_BODY, ARCH_WIDE = 0, 1, 2
PERTURB_EMBEDDING, PERTURB_LSTM, PERTURB_HEAD, PERTURB_ALL = 1, 2, 4, 7

EXPORTS = ("soma_param_count", "soma_workspace_size", "soma_create", "soma_destroy",
           "soma_spsa_step", "soma_spsa_step_adam", "soma_eval_loss", "soma_coefficients",
           "soma_apply_update", "soma_apply_adam", "soma_spsa_step_adam_sched", "soma_schedule_init",
           "soma_schedule_observe", "soma_estimator_moments", "soma_set_tied_head", "soma_head_delta",
           "soma_gaussian", "soma_probe", "soma_philox", "soma_box_muller", "soma_set_phase_timing",
           "soma_get_phase_times", "soma_get_narrow_projections", "soma_set_spin_limit", "soma_spsa_step_noalloc",
           "soma_scan_workspace_size", "soma_scan_forward", "soma_scan_backward", "soma_scan_step",
           "soma_ce_workspace_size", "soma_ce_loss", "soma_ce_grad", "soma_adamw_workspace_size", "soma_adamw_create",
           "soma_adamw_destroy", "soma_adamw_set_rounding", "soma_adamw_step", "soma_adamw_moments", "soma_last_error")


class SomaError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"soma error {code}: {msg}")
        self.code = code


class PhaseTimes(ctypes.Structure):
    _fields_ = [("fold_ms", ctypes.c_float), ("proj_ms", ctypes.c_float),
                ("rec_ms", ctypes.c_float), ("head_ms", ctypes.c_float),
                ("reduce_ms", ctypes.c_float), ("update_ms", ctypes.c_float),
                ("rec_launches", ctypes.c_int32), ("proj_launches", ctypes.c_int32),
                ("xchg_launches", ctypes.c_int32)]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class Adam(ctypes.Structure):
    """soma_adam; the defaults are the paper's (Appendix E)."""
    _fields_ = [("beta1", ctypes.c_float), ("beta2", ctypes.c_float), ("delta", ctypes.c_float),
                ("weight_decay", ctypes.c_float)]

    def __init__(self, beta1=0.9, beta2=0.999, delta=1e-8, weight_decay=1e-4):
        super().__init__(beta1, beta2, delta, weight_decay)


class Plateau(ctypes.Structure):
    """soma_plateau; the defaults are the paper's schedule."""
    _fields_ = [("factor", ctypes.c_float), ("patience", ctypes.c_int32), ("threshold", ctypes.c_float),
                ("floor", ctypes.c_float)]

    def __init__(self, factor=0.5, patience=1000, threshold=1e-8, floor=1e-5):
        super().__init__(factor, patience, threshold, floor)


SCHEDULE_ENTRY_BYTES = 16   # soma_schedule_entry: lr, eps, best (fp32), since (int32)


class Config(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_experts", "n_layers", "embed", "hidden", "batch", "seq_len", "n_pairs", "loss_mode",
        "pair_chunk", "flags", "probe", "accum", "arch")] + [("perturb_mask", ctypes.c_uint32)]


TYPE_FLOAT, TYPE_BFLOAT = 0, 1
SCAN_BLOCK = 32             # rows between the states that a backward scan starts from
ADAMW_BLOCK = 256           # elements that share the scales of 8-bit moments
ROUNDINGS = {"nearest": 0, "random": 1}


class ScanConfig(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("width", ctypes.c_int32), ("sequences", ctypes.c_int32),
                ("type", ctypes.c_int32), ("gate_stride", ctypes.c_int64)]


class CrossEntropyConfig(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_int32), ("vocab", ctypes.c_int32), ("width", ctypes.c_int32),
                ("type", ctypes.c_int32), ("f_stride", ctypes.c_int64), ("e_stride", ctypes.c_int64)]


class AdamWTensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("param", "grad", "m", "v", "m_scale", "v_scale", "copy")] + [
        ("count", ctypes.c_int64), ("weight_decay", ctypes.c_double)] + [
        (n, ctypes.c_int32) for n in ("param_type", "grad_type", "state_bits", "reserved")]


_lib = None


def load():
    """Load libsoma.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: build it with "
                               "`python -m paper_2609_37899_amd.build`")
        lib = ctypes.CDLL(LIB_PATH)
        vp, cp = ctypes.c_void_p, ctypes.POINTER(Config)
        u64, u32, f32, i64p = ctypes.c_uint64, ctypes.c_uint32, ctypes.c_float, ctypes.POINTER(ctypes.c_int64)
        sig = {
            "soma_param_count": (ctypes.c_int, [cp, i64p]),
            "soma_workspace_size": (ctypes.c_int, [cp, ctypes.POINTER(ctypes.c_size_t)]),
            "soma_create": (ctypes.c_int, [cp, vp, ctypes.c_size_t, ctypes.POINTER(vp)]),
            "soma_destroy": (None, [vp]),
            "soma_spsa_step": (ctypes.c_int, [vp, vp, vp, u64, f32, f32, vp, vp, vp]),
            "soma_spsa_step_noalloc": (ctypes.c_int, [cp, vp, vp, u64, f32, f32, vp, vp, vp]),
            "soma_spsa_step_adam": (ctypes.c_int, [vp, vp, vp, vp, ctypes.c_int64, ctypes.POINTER(Adam),
                                                   vp, u64, f32, f32, vp, vp, vp]),
            "soma_apply_adam": (ctypes.c_int, [vp, vp, vp, vp, ctypes.c_int64, ctypes.POINTER(Adam), vp,
                                               u64, f32, vp, vp]),
            "soma_spsa_step_adam_sched": (ctypes.c_int, [vp, vp, vp, vp, ctypes.c_int64, ctypes.POINTER(Adam),
                                                         vp, u64, vp, vp, vp, vp]),
            "soma_schedule_init": (ctypes.c_int, [vp, ctypes.c_int32, f32, f32, vp]),
            "soma_estimator_moments": (ctypes.c_int, [vp, vp, u64, vp, ctypes.c_int32, vp, vp]),
            "soma_schedule_observe": (ctypes.c_int, [vp, ctypes.c_int32, vp, ctypes.c_int32,
                                                     ctypes.POINTER(Plateau), vp]),
            "soma_eval_loss": (ctypes.c_int, [vp, vp, vp, vp, vp]),
            "soma_set_tied_head": (ctypes.c_int, [vp, vp, ctypes.c_int64]),
            "soma_head_delta": (ctypes.c_int, [vp, vp, vp, f32, vp, vp, vp]),
            "soma_coefficients": (ctypes.c_int, [vp, vp, vp]),
            "soma_apply_update": (ctypes.c_int, [vp, vp, vp, u64, f32, vp, vp]),
            "soma_gaussian": (ctypes.c_int, [u64, u64, u32, u64, u64, vp, vp]),
            "soma_probe": (ctypes.c_int, [ctypes.c_int, u64, u64, u32, u64, u64, vp, vp]),
            "soma_philox": (ctypes.c_int, [vp, vp, vp, u64, vp]),
            "soma_box_muller": (ctypes.c_int, [vp, vp, vp, vp, u64, vp]),
            "soma_set_phase_timing": (ctypes.c_int, [vp, ctypes.c_int]),
            "soma_set_spin_limit": (ctypes.c_int, [vp, ctypes.c_uint32]),
            "soma_get_phase_times": (ctypes.c_int, [vp, ctypes.POINTER(PhaseTimes)]),
            "soma_get_narrow_projections": (ctypes.c_int, [vp, ctypes.POINTER(ctypes.c_int32)]),
            "soma_scan_workspace_size": (ctypes.c_int, [ctypes.POINTER(ScanConfig), ctypes.POINTER(ctypes.c_size_t)]),
            "soma_scan_forward": (ctypes.c_int, [ctypes.POINTER(ScanConfig)] + [vp] * 7 + [ctypes.c_size_t, vp]),
            "soma_scan_backward": (ctypes.c_int, [ctypes.POINTER(ScanConfig)] + [vp] * 9 + [ctypes.c_size_t, vp]),
            "soma_scan_step": (ctypes.c_int, [ctypes.POINTER(ScanConfig)] + [vp] * 5),
            "soma_ce_workspace_size": (ctypes.c_int, [ctypes.POINTER(CrossEntropyConfig), ctypes.c_int,
                                                      ctypes.POINTER(ctypes.c_size_t)]),
            "soma_ce_loss": (ctypes.c_int, [ctypes.POINTER(CrossEntropyConfig)] + [vp] * 6 + [ctypes.c_size_t, vp]),
            "soma_ce_grad": (ctypes.c_int, [ctypes.POINTER(CrossEntropyConfig)] + [vp] * 8 + [ctypes.c_size_t, vp]),
            "soma_adamw_workspace_size": (ctypes.c_int, [ctypes.POINTER(AdamWTensor), ctypes.c_int32,
                                                         ctypes.POINTER(ctypes.c_size_t)]),
            "soma_adamw_create": (ctypes.c_int, [ctypes.POINTER(AdamWTensor), ctypes.c_int32, vp, ctypes.c_size_t, vp,
                                                 ctypes.POINTER(vp)]),
            "soma_adamw_destroy": (None, [vp]),
            "soma_adamw_set_rounding": (ctypes.c_int, [vp, ctypes.c_int32, ctypes.c_uint64]),
            "soma_adamw_step": (ctypes.c_int, [vp, ctypes.c_int64] + [ctypes.c_double] * 4 + [vp, vp]),
            "soma_adamw_moments": (ctypes.c_int, [vp, ctypes.POINTER(vp), ctypes.POINTER(vp), vp]),
            "soma_last_error": (ctypes.c_char_p, []),
        }
        for name, (res, args) in sig.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _lib = lib
    return _lib


def _check(rc: int):
    if rc != SOMA_OK:
        raise SomaError(rc, load().soma_last_error().decode())


def _stream(stream=None):
    import torch
    s = stream if stream is not None else torch.cuda.current_stream()
    return ctypes.c_void_p(s.cuda_stream)


def _dptr(t, dtype=None, name="tensor"):
    import torch
    if not isinstance(t, torch.Tensor) or t.device.type != "cuda":
        raise TypeError(f"{name} must be a device tensor")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


@dataclass
class Shape:
    n_experts: int
    n_layers: int
    embed: int
    hidden: int
    batch: int
    seq_len: int
    n_pairs: int
    loss_mode: int = LOSS_INDEPENDENT
    pair_chunk: int = 0
    flags: int = 0
    probe: int = PROBE_GAUSSIAN
    accum: int = 1
    arch: int = ARCH_LSTM
    perturb_mask: int = 0        # PERTURB_* bits of the perturbed groups; 0 = all

    def cfg(self) -> Config:
        return Config(self.n_experts, self.n_layers, self.embed, self.hidden, self.batch,
                      self.seq_len, self.n_pairs, self.loss_mode, self.pair_chunk, self.flags,
                      self.probe, self.accum, self.arch, self.perturb_mask)

    @property
    def directions(self) -> int:
        """Directions per update, n_pairs per accumulation batch."""
        return self.n_pairs * max(1, self.accum)


def param_count(shape: Shape) -> int:
    out = ctypes.c_int64()
    _check(load().soma_param_count(ctypes.byref(shape.cfg()), ctypes.byref(out)))
    return out.value


def workspace_size(shape: Shape) -> int:
    out = ctypes.c_size_t()
    _check(load().soma_workspace_size(ctypes.byref(shape.cfg()), ctypes.byref(out)))
    return out.value


class Context:
    """A shape bound to a device workspace (a torch uint8 tensor)."""

    def __init__(self, shape: Shape, device="cuda"):
        import torch
        self.shape = shape
        self._cfg = shape.cfg()
        nbytes = workspace_size(shape)
        self.workspace = torch.empty(max(nbytes, 256), dtype=torch.uint8, device=device)
        h = ctypes.c_void_p()
        _check(load().soma_create(ctypes.byref(self._cfg), ctypes.c_void_p(self.workspace.data_ptr()),
                                  nbytes, ctypes.byref(h)))
        self._h = h
        self.d = param_count(shape)

    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            load().soma_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def spsa_step(self, theta, seeds, step: int, eps: float, lr: float, bytes_, losses,
                  stream=None):
        import torch
        _check(load().soma_spsa_step(self._h, _dptr(theta, torch.float32, "theta"),
                                     _dptr(seeds, torch.int64, "seeds"), int(step), float(eps),
                                     float(lr), _dptr(bytes_, torch.uint8, "bytes"),
                                     _dptr(losses, torch.float32, "losses"), _stream(stream)))

    def spsa_step_adam(self, theta, m, v, t: int, adam, seeds, step: int, eps: float, lr: float, bytes_,
                       losses, stream=None):
        import torch
        _check(load().soma_spsa_step_adam(self._h, _dptr(theta, torch.float32, "theta"),
                                          _dptr(m, torch.float32, "m"), _dptr(v, torch.float32, "v"),
                                          int(t), ctypes.byref(adam), _dptr(seeds, torch.int64, "seeds"),
                                          int(step), float(eps), float(lr),
                                          _dptr(bytes_, torch.uint8, "bytes"),
                                          _dptr(losses, torch.float32, "losses"), _stream(stream)))

    def spsa_step_adam_sched(self, theta, m, v, t: int, adam, seeds, step: int, sched, bytes_, losses,
                             stream=None):
        import torch
        _check(load().soma_spsa_step_adam_sched(self._h, _dptr(theta, torch.float32, "theta"),
                                                _dptr(m, torch.float32, "m"), _dptr(v, torch.float32, "v"),
                                                int(t), ctypes.byref(adam), _dptr(seeds, torch.int64, "seeds"),
                                                int(step), _dptr(sched, None, "schedule"),
                                                _dptr(bytes_, torch.uint8, "bytes"),
                                                _dptr(losses, torch.float32, "losses"), _stream(stream)))

    def estimator_moments(self, seeds, step: int, coef, group: int, out, stream=None):
        import torch
        _check(load().soma_estimator_moments(self._h, _dptr(seeds, torch.int64, "seeds"), int(step),
                                             _dptr(coef, torch.float32, "coef"), int(group),
                                             _dptr(out, torch.float64, "out"), _stream(stream)))

    def apply_adam(self, theta, m, v, t: int, adam, seeds, step: int, lr: float, coef, stream=None):
        import torch
        _check(load().soma_apply_adam(self._h, _dptr(theta, torch.float32, "theta"),
                                      _dptr(m, torch.float32, "m"), _dptr(v, torch.float32, "v"), int(t),
                                      ctypes.byref(adam), _dptr(seeds, torch.int64, "seeds"), int(step),
                                      float(lr), _dptr(coef, torch.float32, "coef"), _stream(stream)))

    def set_phase_timing(self, enable: bool = True):
        _check(load().soma_set_phase_timing(self._h, 1 if enable else 0))

    def set_spin_limit(self, polls: int):
        """Polls per group barrier of the persistent recurrence (0: default)."""
        _check(load().soma_set_spin_limit(self._h, int(polls)))

    def narrow_projections(self) -> int:
        out = ctypes.c_int32()
        _check(load().soma_get_narrow_projections(self._h, ctypes.byref(out)))
        return out.value

    def phase_times(self) -> dict:
        out = PhaseTimes()
        _check(load().soma_get_phase_times(self._h, ctypes.byref(out)))
        return out.as_dict()

    def eval_loss(self, theta, bytes_, loss, stream=None):
        import torch
        _check(load().soma_eval_loss(self._h, _dptr(theta, torch.float32, "theta"),
                                     _dptr(bytes_, torch.uint8, "bytes"),
                                     _dptr(loss, torch.float32, "loss"), _stream(stream)))

    def set_tied_head(self, E, per_expert: bool = False):
        """The tied matrix of a body context: E [V][w] shared by every expert,
        or [N][V][w] one per expert (per_expert=True); w = d, or d_E for the
        wide body.  The context reads the tensor's memory on every later
        call: keep it alive."""
        import torch
        stride = E.shape[-2] * E.shape[-1] if per_expert else 0
        _check(load().soma_set_tied_head(self._h, _dptr(E, torch.float32, "E"), stride))
        self._head = E

    def head_delta(self, theta, bytes_, lr: float = 0.0, grad=None, loss=None, stream=None):
        """The decoder-path delta rule: grad [N][V][d] and loss [N] (either may
        be None); with lr != 0 the tied matrix is also moved by -lr grad."""
        import torch
        g = _dptr(grad, torch.float32, "grad") if grad is not None else None
        lo = _dptr(loss, torch.float32, "loss") if loss is not None else None
        _check(load().soma_head_delta(self._h, _dptr(theta, torch.float32, "theta"),
                                      _dptr(bytes_, torch.uint8, "bytes"), float(lr), g, lo, _stream(stream)))

    def coefficients(self, coef, stream=None):
        import torch
        _check(load().soma_coefficients(self._h, _dptr(coef, torch.float32, "coef"), _stream(stream)))

    def apply_update(self, theta, seeds, step: int, lr: float, coef, stream=None):
        import torch
        _check(load().soma_apply_update(self._h, _dptr(theta, torch.float32, "theta"),
                                        _dptr(seeds, torch.int64, "seeds"), int(step), float(lr),
                                        _dptr(coef, torch.float32, "coef"), _stream(stream)))


def spsa_step_noalloc(shape: Shape, theta, seeds, step: int, eps: float, lr: float, bytes_, losses, stream=None):
    """soma_spsa_step without a context or workspace: the library's static
    per-device scratch (small shapes only; calls on one GPU must not overlap)."""
    import torch
    cfg = shape.cfg()
    _check(load().soma_spsa_step_noalloc(ctypes.byref(cfg), _dptr(theta, torch.float32, "theta"),
                                         _dptr(seeds, torch.int64, "seeds"), int(step), float(eps), float(lr),
                                         _dptr(bytes_, torch.uint8, "bytes"), _dptr(losses, torch.float32, "losses"),
                                         _stream(stream)))


def gaussian(seed: int, step: int, pair: int, k0: int, out, stream=None):
    import torch
    _check(load().soma_gaussian(int(seed) & (2**64 - 1), int(step), int(pair), int(k0), out.numel(),
                                _dptr(out, torch.float32, "out"), _stream(stream)))


def probe(law: int, seed: int, step: int, pair: int, k0: int, out, stream=None):
    import torch
    _check(load().soma_probe(int(law), int(seed) & (2**64 - 1), int(step), int(pair), int(k0), out.numel(),
                             _dptr(out, torch.float32, "out"), _stream(stream)))


def schedule_tensor(n: int, device="cuda"):
    """Device memory for n soma_schedule_entry records (int32 view, 4 words each)."""
    import torch
    return torch.empty((n, SCHEDULE_ENTRY_BYTES // 4), dtype=torch.int32, device=device)


def schedule_init(sched, lr0: float, eps0: float, stream=None):
    _check(load().soma_schedule_init(_dptr(sched, None, "schedule"), sched.shape[0], float(lr0), float(eps0),
                                     _stream(stream)))


def schedule_observe(sched, val_loss, updates: int, rule, stream=None):
    import torch
    _check(load().soma_schedule_observe(_dptr(sched, None, "schedule"), sched.shape[0],
                                        _dptr(val_loss, torch.float32, "val_loss"), int(updates),
                                        ctypes.byref(rule), _stream(stream)))


def schedule_fields(sched):
    """(lr, eps, best, since) numpy arrays of a schedule tensor (copies to the host)."""
    import numpy as np
    a = sched.cpu().numpy()
    f = a.view(np.float32)
    return f[:, 0].copy(), f[:, 1].copy(), f[:, 2].copy(), a[:, 3].copy()


def philox(ctr, key, out, stream=None):
    import torch
    n = ctr.shape[0]
    _check(load().soma_philox(_dptr(ctr, torch.int32, "ctr"), _dptr(key, torch.int32, "key"),
                              _dptr(out, torch.int32, "out"), n, _stream(stream)))


def box_muller(wa, wb, za, zb, stream=None):
    import torch
    _check(load().soma_box_muller(_dptr(wa, torch.int32, "wa"), _dptr(wb, torch.int32, "wb"),
                                  _dptr(za, torch.float32, "za"), _dptr(zb, torch.float32, "zb"),
                                  wa.numel(), _stream(stream)))


def group_covariance_trace(moments, directions: int, group: int):
    """tr Cov of the group means of `group` consecutive single-direction
    estimates, from soma_estimator_moments' two sums (per expert)."""
    import numpy as np
    m = np.asarray(moments, dtype=np.float64).reshape(-1, 2)
    G = directions // group
    return (m[:, 0] - m[:, 1] / G) / (group * group * (G - 1))


def seeds_tensor(seeds, device="cuda"):
    """uint64 seeds as the int64 device tensor the library reads bit for bit."""
    import numpy as np
    import torch
    a = np.ascontiguousarray(seeds, dtype=np.uint64).view(np.int64)
    return torch.from_numpy(a.copy()).to(device)


# ---------------------------------------------------------------------------
# Operators of first-order training

def _type_of(dtype) -> int:
    import torch
    if dtype == torch.float32:
        return TYPE_FLOAT
    if dtype == torch.bfloat16:
        return TYPE_BFLOAT
    raise TypeError(f"dtype must be torch.float32 or torch.bfloat16, got {dtype}")


class _Plan:
    """What the operators' classes share: one device, a workspace on it, and
    the checks of their arguments.  A plan must not be used by two streams at
    once, nor by two captured graphs that may run at once: its workspace is
    shared.  A captured graph holds the addresses of the plan's memory, not the
    plan: keep the plan as long as the graph."""

    def _start(self, nbytes: int, device):
        import torch
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise TypeError("device must be a GPU")
        if self.device.index is None:
            self.device = torch.device("cuda", torch.cuda.current_device())
        self.workspace = torch.empty(max(int(nbytes), 256), dtype=torch.uint8, device=self.device)
        self._memory = [self.workspace]
        st = torch.cuda.current_stream(self.device)
        self._stream0 = st.cuda_stream
        if not torch.cuda.is_current_stream_capturing():
            st.synchronize()           # other streams may use the memory as well: nothing before is under way in it
        self._ws = ctypes.c_void_p(self.workspace.data_ptr())

    def _call(self, stream, fn, *args):
        """fn(*args, stream) with the plan's device current."""
        import torch
        st = stream if stream is not None else torch.cuda.current_stream(self.device)
        raw = st.cuda_stream
        if stream is not None and st.device != self.device:
            raise ValueError(f"stream belongs to {st.device}, the plan to {self.device}")
        if raw != self._stream0:
            for x in self._memory:
                x.record_stream(st)                   # not handed out again before this stream is done with it
        if torch.cuda.current_device() == self.device.index:
            rc = fn(*args, raw)
        else:
            with torch.cuda.device(self.device):
                rc = fn(*args, raw)
        if rc != SOMA_OK:
            _check(rc)

    def _ptr(self, t, name, dtype, shape, optional=False, strided=False):
        """The address of a tensor of this type and shape on the plan's device
        (strided: rows may lie further apart than their length)."""
        import torch
        if t is None and optional:
            return None
        # get_device() is -1 for the CPU
        if not isinstance(t, torch.Tensor) or t.get_device() != self.device.index or t.device.type != "cuda":
            raise TypeError(f"{name} must be a tensor on {self.device}")
        if t.dtype != dtype:
            raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
        if t.shape != shape:
            raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
        if not t.is_contiguous():
            if not strided or t.dim() != 2:
                raise ValueError(f"{name} must be contiguous")
            if t.shape[1] > 1 and t.stride(1) != 1 or t.shape[0] > 1 and t.stride(0) < t.shape[1]:
                raise ValueError(f"{name} must have contiguous rows that do not overlap")
        return t.data_ptr()


def _row_stride(t) -> int:
    """Elements between rows (of one row, its length)."""
    return t.stride(0) if t.shape[0] > 1 else t.shape[1]


def _check_sizes(**sizes):
    for name, n in sizes.items():
        if not 0 <= n < 2**31:
            raise ValueError(f"{name} must be in [0, 2^31)")


class GatedScan(_Plan):
    """The gated linear recurrence: the LSTM's cell with gates that read the
    input alone, c_t = s(f_t) c_{t-1} + s(i_t) tanh(g_t), h_t = s(o_t) tanh(c_t),
    over ``sequences`` sequences that lie behind one another in at most ``rows``
    rows of ``width`` channels.  ``dtype`` (float32 or bfloat16) is the type of
    gates, h and their gradients; states are float32.

    gates [n][4 width] hold the pre-activations in blocks i, f, g, o; rows may be
    strided.  offsets [sequences + 1] (int32, on the device) gives each
    sequence's first row; None: all sequences have n / sequences rows.  Rows
    behind the last sequence are neither read nor written.  A sequence far longer
    than the others of its batch is best given a call of its own (soma.h)."""

    def __init__(self, rows: int, sequences: int, width: int, dtype, device="cuda"):
        self.rows, self.sequences, self.width, self.dtype = int(rows), int(sequences), int(width), dtype
        self._type = _type_of(dtype)
        _check_sizes(rows=self.rows, sequences=self.sequences, width=self.width)
        out = ctypes.c_size_t()
        _check(load().soma_scan_workspace_size(ctypes.byref(self._cfg(self.rows, 4 * self.width)), ctypes.byref(out)))
        self._bytes = out.value
        self._start(out.value, device)

    def _cfg(self, rows, stride):
        return ScanConfig(rows, self.width, self.sequences, self._type, stride)

    def new_states(self):
        """An array for forward's states (what backward starts from)."""
        import torch
        return torch.empty((-(-self.rows // SCAN_BLOCK), self.width), dtype=torch.float32, device=self.device)

    def _gates(self, gates, offsets):
        import torch
        if not isinstance(gates, torch.Tensor) or gates.dim() != 2:
            raise TypeError("gates must be a tensor [rows][4 width]")
        n = gates.shape[0]
        if n > self.rows:
            raise ValueError(f"{n} rows, but the plan was made for {self.rows}")
        return (n, self._cfg(n, _row_stride(gates)), self._ptr(gates, "gates", self.dtype, (n, 4 * self.width), strided=True),
                self._ptr(offsets, "offsets", torch.int32, (self.sequences + 1,), optional=True))

    def _states(self, states, n, optional):
        import torch
        if states is None and optional:
            return None
        if not isinstance(states, torch.Tensor) or states.dim() != 2 or states.shape[0] < -(-n // SCAN_BLOCK):
            raise ValueError(f"states must be a tensor of {-(-n // SCAN_BLOCK)} rows or more (new_states())")
        return self._ptr(states, "states", torch.float32, (states.shape[0], self.width))

    def forward(self, gates, h, c0=None, cT=None, states=None, offsets=None, stream=None):
        """h [n][width] from gates; cT [sequences][width] receives the states
        behind the last rows (it may be c0), states what backward needs."""
        import torch
        n, cfg, pg, po = self._gates(gates, offsets)
        end = (self.sequences, self.width)
        self._call(stream, load().soma_scan_forward, ctypes.byref(cfg), pg, po,
                   self._ptr(c0, "c0", torch.float32, end, optional=True), self._ptr(h, "h", self.dtype, (n, self.width)),
                   self._ptr(cT, "cT", torch.float32, end, optional=True), self._states(states, n, True), self._ws,
                   self._bytes)

    def backward(self, gates, states, dh, dgates, c0=None, dcT=None, dc0=None, offsets=None, stream=None):
        """dgates [n][4 width] and dc0 from dh [n][width] and dcT, with the
        gates, offsets and c0 that forward had and the states it gave."""
        import torch
        n, cfg, pg, po = self._gates(gates, offsets)
        end = (self.sequences, self.width)
        self._call(stream, load().soma_scan_backward, ctypes.byref(cfg), pg, po,
                   self._ptr(c0, "c0", torch.float32, end, optional=True), self._states(states, n, False),
                   self._ptr(dh, "dh", self.dtype, (n, self.width)),
                   self._ptr(dcT, "dcT", torch.float32, end, optional=True),
                   self._ptr(dgates, "dgates", self.dtype, (n, 4 * self.width)),
                   self._ptr(dc0, "dc0", torch.float32, end, optional=True), self._ws, self._bytes)

    def step(self, gates, c0, cT, h, stream=None):
        """One row for every sequence: cT (it may be c0) and h [sequences][width]."""
        import torch
        n, cfg, pg, _ = self._gates(gates, None)
        end = (self.sequences, self.width)
        self._call(stream, load().soma_scan_step, ctypes.byref(cfg), pg,
                   self._ptr(c0, "c0", torch.float32, end, optional=True), self._ptr(cT, "cT", torch.float32, end),
                   self._ptr(h, "h", self.dtype, end))


class CrossEntropy(_Plan):
    """Softmax cross entropy of a linear head, logits f E^T, for at most ``rows``
    rows f [n][width] and a head E [vocab][width] of ``dtype`` (float32 or
    bfloat16; rows may be strided), without the logits in memory.  targets [n]
    int32; a row with a negative one counts for nothing.  grad: gradients are
    wanted too (a larger workspace)."""

    def __init__(self, rows: int, vocab: int, width: int, dtype, grad: bool = True, device="cuda"):
        self.rows, self.vocab, self.width, self.dtype, self.with_grad = int(rows), int(vocab), int(width), dtype, bool(grad)
        self._type = _type_of(dtype)
        _check_sizes(rows=self.rows, vocab=self.vocab, width=self.width)
        out = ctypes.c_size_t()
        cfg = CrossEntropyConfig(self.rows, self.vocab, self.width, self._type, self.width, self.width)
        _check(load().soma_ce_workspace_size(ctypes.byref(cfg), int(self.with_grad), ctypes.byref(out)))
        self._bytes = out.value
        self._start(out.value, device)

    def _inputs(self, f, E, targets):
        import torch
        if not isinstance(f, torch.Tensor) or f.dim() != 2:
            raise TypeError("f must be a tensor [rows][width]")
        n = f.shape[0]
        if n > self.rows:
            raise ValueError(f"{n} rows, but the plan was made for {self.rows}")
        pf = self._ptr(f, "f", self.dtype, (n, self.width), strided=True)
        pe = self._ptr(E, "E", self.dtype, (self.vocab, self.width), strided=True)
        cfg = CrossEntropyConfig(n, self.vocab, self.width, self._type, _row_stride(f), _row_stride(E))
        return n, cfg, pf, pe, self._ptr(targets, "targets", torch.int32, (n,))

    def loss(self, f, E, targets, loss, lse=None, stream=None):
        """loss [n] and lse [n] (float32): the rows' cross entropies in nats and
        log-sum-exps."""
        import torch
        n, cfg, pf, pe, pt = self._inputs(f, E, targets)
        self._call(stream, load().soma_ce_loss, ctypes.byref(cfg), pf, pe, pt,
                   self._ptr(loss, "loss", torch.float32, (n,), optional=True),
                   self._ptr(lse, "lse", torch.float32, (n,), optional=True), self._ws, self._bytes)

    def grad(self, f, E, targets, lse, grad_loss, df=None, dE=None, stream=None):
        """df [n][width] and dE [vocab][width] (either may be None) of
        sum(grad_loss * loss), with the lse that loss() gave."""
        import torch
        if not self.with_grad:
            raise ValueError("the plan was made without gradients")
        n, cfg, pf, pe, pt = self._inputs(f, E, targets)
        self._call(stream, load().soma_ce_grad, ctypes.byref(cfg), pf, pe, pt,
                   self._ptr(lse, "lse", torch.float32, (n,)), self._ptr(grad_loss, "grad_loss", torch.float32, (n,)),
                   self._ptr(df, "df", self.dtype, (n, self.width), optional=True),
                   self._ptr(dE, "dE", self.dtype, (self.vocab, self.width), optional=True), self._ws, self._bytes)


class AdamW(_Plan):
    """AdamW over many tensors in one launch.  params and grads are lists of
    contiguous tensors (float32 or bfloat16, a pair may differ), whose memory the
    plan uses at every step: keep them in place.  bits: moments in 32 or in 8.
    weight_decay: one value, or one for each tensor.  moments: a list of (m, v),
    or for 8 bits (m, v, m_scale, v_scale), to go on from; None: zeros.  copies:
    bfloat16 tensors (or None) that receive the new parameters too.

    rounding of moments in 8 bits: "random" for a training run, drawn from seed
    and the update's number, or "nearest", the closest codes of a single step.  To
    nearest, v does not follow its average over many steps, since updates of less
    than half a code (3 to 6% of v) are lost."""

    def __init__(self, params, grads, bits: int = 32, weight_decay=0.01, betas=(0.9, 0.999), delta: float = 1e-8,
                 moments=None, copies=None, stream=None, rounding: str = "nearest", seed: int = 0):
        import torch
        self._h = ctypes.c_void_p()
        params, grads = list(params), list(grads)
        n = len(params)
        copies = list(copies) if copies is not None else [None] * n
        decay = list(weight_decay) if isinstance(weight_decay, (list, tuple)) else [weight_decay] * n
        if n == 0 or len(grads) != n or len(copies) != n or len(decay) != n:
            raise ValueError("params must not be empty; grads, copies and weight_decay must be as many")
        if bits not in (8, 32):
            raise ValueError("bits must be 8 or 32")
        if rounding not in ROUNDINGS:
            raise ValueError(f"rounding must be one of {sorted(ROUNDINGS)}")
        if not isinstance(params[0], torch.Tensor) or params[0].device.type != "cuda":
            raise TypeError("params must be device tensors")
        self.device, self.bits, self.betas, self.delta = params[0].device, bits, tuple(betas), float(delta)
        state = torch.float32 if bits == 32 else torch.uint8
        self._own = None
        if moments is None:
            # one allocation, every array 256 bytes aligned
            sizes = []
            for p in params:
                blocks = -(-p.numel() // ADAMW_BLOCK)
                sizes += [p.numel()] * 2 if bits == 32 else [p.numel(), p.numel(), blocks, blocks]
            types = [torch.float32] * 2 if bits == 32 else [torch.uint8, torch.uint8, torch.float32, torch.float32]
            ends, end = [], 0
            for i, k in enumerate(sizes):
                end = -(-(end + k * types[i % len(types)].itemsize) // 256) * 256
                ends.append(end)
            self._own = torch.zeros(end, dtype=torch.uint8, device=self.device)
            arrays = [self._own[at:at + k * types[i % len(types)].itemsize].view(types[i % len(types)])
                      for i, (at, k) in enumerate(zip([0] + ends, sizes))]
            moments = [tuple(arrays[i:i + len(types)]) for i in range(0, len(arrays), len(types))]
        self.state = [tuple(x) for x in moments]
        if len(self.state) != n or any(len(x) != (2 if bits == 32 else 4) for x in self.state):
            raise ValueError("moments must hold (m, v) for each tensor, or (m, v, m_scale, v_scale) for 8 bits")
        table = (AdamWTensor * n)()
        for i, (p, g, x, c, w) in enumerate(zip(params, grads, self.state, copies, decay)):
            at = f"params[{i}]"
            pp = self._ptr(p, at, p.dtype if isinstance(p, torch.Tensor) else None, p.shape)
            pg = self._ptr(g, f"grads[{i}]", g.dtype if isinstance(g, torch.Tensor) else None, p.shape)
            px = [self._ptr(t.view(-1) if t.is_contiguous() else t, f"moments[{i}]", d, (k,))
                  for t, d, k in zip(x, (state, state, torch.float32, torch.float32),
                                     (p.numel(), p.numel()) + (-(-p.numel() // ADAMW_BLOCK),) * 2)]
            px += [None] * (4 - len(px))
            table[i] = AdamWTensor(pp, pg, *px, self._ptr(c, f"copies[{i}]", torch.bfloat16, p.shape, optional=True),
                                   p.numel(), float(w), _type_of(p.dtype), _type_of(g.dtype), bits, 0)
        self.params, self.grads, self.copies = params, grads, copies
        self._shapes = [p.shape for p in params]
        out = ctypes.c_size_t()
        _check(load().soma_adamw_workspace_size(table, n, ctypes.byref(out)))
        self._start(out.value, self.device)
        if self._own is not None:
            self._memory.append(self._own)
        plan = ctypes.c_void_p()
        with torch.cuda.device(self.device):
            st = stream if stream is not None else torch.cuda.current_stream(self.device)
            _check(load().soma_adamw_create(table, n, self._ws, out.value, ctypes.c_void_p(st.cuda_stream),
                                            ctypes.byref(plan)))
        self._h = plan
        self.rounding, self.seed = rounding, int(seed)
        _check(load().soma_adamw_set_rounding(plan, ROUNDINGS[rounding], self.seed & (2**64 - 1)))

    def close(self):
        if self._h.value:
            load().soma_adamw_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def step(self, t: int, lr: float, grad_scale=None, stream=None):
        """Update number t >= 1.  grad_scale: one float32 value on the device
        that every gradient is multiplied with (None: 1).  A captured step repeats
        its t, its lr and its random rounding at every replay."""
        import torch
        if not self._h.value:
            raise RuntimeError("the plan is closed")
        if grad_scale is not None:
            grad_scale = self._ptr(grad_scale.view(-1) if isinstance(grad_scale, torch.Tensor) else grad_scale,
                                   "grad_scale", torch.float32, (1,))
        self._call(stream, load().soma_adamw_step, self._h, int(t), float(lr), float(self.betas[0]),
                   float(self.betas[1]), self.delta, grad_scale)

    def moments(self, m_out, v_out, stream=None):
        """The values of the moments, in float32: lists of tensors as large as
        the parameters."""
        import torch
        if not self._h.value:
            raise RuntimeError("the plan is closed")
        n = len(self.params)
        if len(m_out) != n or len(v_out) != n:
            raise ValueError(f"m_out and v_out must hold {n} tensors")
        arrays, index = [], self.device.index
        for name, x in (("m_out", m_out), ("v_out", v_out)):
            for i, (t, shape) in enumerate(zip(x, self._shapes)):
                # hundreds of tensors: the full check, a microsecond each, only for what is not plainly right
                if not (isinstance(t, torch.Tensor) and t.dtype is torch.float32 and t.get_device() == index
                        and t.shape == shape and t.is_contiguous()):
                    self._ptr(t, f"{name}[{i}]", torch.float32, shape)
            arrays.append((ctypes.c_void_p * n)(*[t.data_ptr() for t in x]))
        self._call(stream, load().soma_adamw_moments, self._h, *arrays)
