"""ctypes binding of libsd_mi355x.so -- argument marshalling only.

Every function here has the name of the C entry point it forwards to (``include/sd.h``,
``include/sdden.h``).  PyTorch is used for device memory and streams: tensors are checked for
device / dtype / contiguity and their raw pointers handed to the library.  There is no
fallback: if the shared library is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes
import os
from ctypes import POINTER, c_char_p, c_float, c_int, c_int32, c_int64, c_size_t, c_uint64, c_void_p
from typing import Optional

import numpy as np
import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libsd_mi355x.so")

SD_DRAFT_FROZEN = 0
SD_DRAFT_EXPLICIT = 1
SD_DRAFT_FROZEN_REUSED = 2
SD_MAX_WINDOW = 64
SD_STATIC_MAX_CHAINS = 65536
SD_CARRY_DRAFT = 0
SD_CARRY_LAST_ACCEPTED = 1
SD_ERR_UNSUPPORTED = -5
SDDEN_F32 = 0
SDDEN_BF16 = 1
SDDEN_SILU = 0
SDDEN_GELU = 1


class SDError(RuntimeError):
    pass


class _Schedule(ctypes.Structure):
    _fields_ = [("T", c_int32), ("a", POINTER(c_float)), ("c", POINTER(c_float)),
                ("sigma", POINTER(c_float))]


_SIGNATURES = {
    # sd.h
    "sd_create": (c_int, [POINTER(_Schedule), c_int32, c_int32, POINTER(c_void_p)]),
    "sd_destroy": (c_int, [c_void_p]),
    "sd_set_seed": (c_int, [c_void_p, c_uint64]),
    "sd_set_draft_mode": (c_int, [c_void_p, c_int]),
    "sd_set_temperature": (c_int, [c_void_p, c_float]),
    "sd_set_active_count": (c_int, [c_void_p, c_void_p]),
    "sd_set_verify_shape": (c_int, [c_void_p, c_int32]),
    "sd_workspace_bytes": (c_size_t, [c_void_p, c_int32]),
    "sd_set_workspace": (c_int, [c_void_p, c_void_p, c_size_t]),
    "sd_init_state": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p]),
    "sd_draft": (c_int, [c_void_p, c_int32] + [c_void_p] * 7),
    "sd_draft_step": (c_int, [c_void_p, c_int32, c_int32] + [c_void_p] * 10),
    "sd_set_start_prediction": (c_int, [c_void_p, c_void_p]),
    "sd_set_carry": (c_int, [c_void_p, c_void_p, c_void_p]),
    "sd_set_carry_rule": (c_int, [c_void_p, c_int32]),
    "sd_set_draft_mirror": (c_int, [c_void_p, c_void_p]),
    "sdden_eval_mirror": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p]),
    "sd_verify": (c_int, [c_void_p, c_int32] + [c_void_p] * 12),
    "sd_advance": (c_int, [c_void_p, c_int32] + [c_void_p] * 10),
    "sd_advance_static": (c_int, [c_void_p, c_int32] + [c_void_p] * 10),
    "sd_langevin_window": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_float, c_int32, c_float] + [c_void_p] * 6),
    "sd_langevin_window_phi4": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_float, c_float]
                                + [c_void_p] * 6),
    "sd_langevin_chains": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                   c_float, c_int32, c_float, c_void_p, c_void_p, c_void_p, c_void_p]),
    "sd_langevin_run": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p, c_void_p,
                                c_float, c_int32, c_float, c_int32] + [c_void_p] * 4),
    "sd_langevin_run_phi4": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_float, c_float,
                                     c_int32] + [c_void_p] * 4),
    "sd_last_error": (c_char_p, [c_void_p]),
    # sd_measure.h
    "sd_measure_stream": (c_int, [c_void_p, c_void_p, c_size_t, c_int32, c_int32, c_void_p]),
    "sd_measure_mfma": (c_int, [c_int32, c_int32, c_int32, c_void_p, POINTER(ctypes.c_double), c_void_p]),
    # sdden.h
    "sdden_gmm_create": (c_int, [c_int32, c_int32, c_void_p, c_void_p, c_void_p, c_int32, c_void_p,
                                 POINTER(c_void_p)]),
    "sdden_lowrank_create": (c_int, [c_int32, c_int32, c_void_p, c_void_p, c_float, c_int32, c_void_p,
                                     POINTER(c_void_p)]),
    "sdden_mlp_create": (c_int, [c_int32, c_int32, c_int32] + [c_void_p] * 6 + [c_int32, c_int32,
                                                                               POINTER(c_void_p)]),
    "sdden_mlp4_create": (c_int, [c_int32] * 4 + [c_void_p] * 6 + [c_int32, c_int32, POINTER(c_void_p)]),
    "sdden_gated_create": (c_int, [c_int32] * 5 + [c_void_p] * 4 + [c_float] + [c_void_p] * 3 + [c_int32, c_int32, POINTER(c_void_p)]),
    "sdden_reserve": (c_int, [c_void_p, c_int32]),
    "sdden_eval": (c_int, [c_void_p, c_int32, c_void_p, c_void_p, c_void_p, c_void_p]),
    "sdden_run": (c_int, [c_void_p, c_void_p, c_void_p, c_int32] + [c_void_p] * 8),
    "sdden_set_active_count": (c_int, [c_void_p, c_void_p, c_int32]),
    "sdden_profile": (c_int, [c_void_p, c_int32]),
    "sdden_profile_min_rows": (c_int, [c_void_p, c_int32]),
    "sdden_profile_collect": (c_int, [c_void_p, POINTER(ctypes.c_double), POINTER(c_int64)]),
    "sdden_mlp_select_gemm": (c_int, [c_void_p, c_int32]),
    "sdden_destroy": (c_int, [c_void_p]),
    "sdden_last_error": (c_char_p, [c_void_p]),
    "sdden_layernorm_workspace_bytes": (c_size_t, [c_int32, c_int32]),
    "sdden_layernorm_forward": (c_int, [c_int32, c_int32, c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_float, c_void_p, c_int32,
                                        c_int64, c_void_p, c_void_p, c_void_p]),
    "sdden_layernorm_backward": (c_int, [c_int32, c_int32, c_void_p, c_int32, c_int64, c_void_p, c_int32, c_int64, c_void_p, c_void_p,
                                         c_void_p, c_void_p, c_int64, c_void_p, c_int64, c_void_p, c_void_p, c_void_p, c_size_t,
                                         c_void_p]),
    "sdden_q4_create": (c_int, [c_int32] * 3 + [c_void_p] * 2 + [POINTER(c_void_p)]),
    "sdden_q4_eval": (c_int, [c_void_p, c_int32, c_void_p, c_int32, c_int64, c_void_p, c_void_p, c_int32, c_int64, c_void_p]),
    "sdden_q4_destroy": (c_int, [c_void_p]),
    "sdden_gated_workspace_bytes": (c_size_t, [c_int32, c_int32, c_int32]),
    "sdden_gated_forward": (c_int, [c_int32] * 4 + [c_void_p, c_int64] + [c_void_p] * 5 + [c_int32, c_int64] + [c_void_p] * 3),
    "sdden_gated_backward": (c_int, [c_int32] * 4 + [c_void_p, c_int64, c_void_p, c_int64] + [c_void_p] * 6 + [c_int64]
                             + [c_void_p] * 3 + [c_int32, c_void_p, c_size_t, c_void_p]),
}

_lib = None


def exported_symbols():
    """Names the headers declare (and the binding expects)."""
    return sorted(_SIGNATURES)


def load_library(path: Optional[str] = None):
    """dlopen the HIP library; raises SDError when it has not been built."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise SDError(f"{p} not found: build it first (python -m paper_2501_05370_amd.build). "
                      "There is no CPU fallback.")
    lib = ctypes.CDLL(p)
    for name, (res, args) in _SIGNATURES.items():
        fn = getattr(lib, name)            # AttributeError if a declared symbol is not exported
        fn.restype, fn.argtypes = res, args
    if path is None:
        _lib = lib
    return lib


def _stream() -> int:
    """Handle of torch's current stream on the current device, read from torch's runtime directly: the Stream object that
    ``torch.cuda.current_stream()`` builds for every call costs 2.5 us, and calls on few chains are bound by the host.  Draft
    and two low-rank predictions for 19 chains: 32 us a pass, 37.7 with it; accept calls on 8 chains 27 and 33.  Looked up
    at the call: a torch built without GPU support has neither function, and can still import this module."""
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


def _dev(t: Optional[torch.Tensor], dtype, name: str, allow_none: bool = False) -> Optional[int]:
    if t is None:
        if allow_none:
            return None
        raise SDError(f"{name}: tensor required")
    if t.is_cuda and t.dtype is dtype and t.is_contiguous():
        return t.data_ptr()
    raise SDError(f"{name}: need a contiguous {dtype} CUDA tensor, got {t.dtype} on {t.device}, "
                  f"contiguous={t.is_contiguous()}")


def _host(a, dtype) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(a), dtype=dtype)


class Context:
    """Owns one ``sd_ctx``.  Methods are the C calls with tensors in place of pointers."""

    def __init__(self, a, c, sigma, d: int, K: int):
        self._lib = load_library()
        self._a, self._c, self._s = _host(a, np.float32), _host(c, np.float32), _host(sigma, np.float32)
        T = self._a.shape[0]
        if self._c.shape[0] != T or self._s.shape[0] != T:
            raise SDError("schedule arrays must have the same length")
        sch = _Schedule(T, self._a.ctypes.data_as(POINTER(c_float)), self._c.ctypes.data_as(POINTER(c_float)),
                        self._s.ctypes.data_as(POINTER(c_float)))
        h = c_void_p()
        rc = self._lib.sd_create(ctypes.byref(sch), d, K, ctypes.byref(h))
        if rc != 0:
            raise SDError(f"sd_create failed ({rc}): {self._lib.sd_last_error(None).decode()}")
        self._h = h
        self.T, self.d, self.K = T, d, K
        self._ws = None
        self._keep = []

    def close(self):
        if getattr(self, "_h", None):
            self._lib.sd_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, rc: int, what: str):
        if rc != 0:
            raise SDError(f"{what} failed ({rc}): {self._lib.sd_last_error(self._h).decode()}")

    # -- setters
    def sd_set_seed(self, seed: int):
        self._check(self._lib.sd_set_seed(self._h, seed), "sd_set_seed")

    def sd_set_draft_mode(self, mode: int):
        self._check(self._lib.sd_set_draft_mode(self._h, mode), "sd_set_draft_mode")

    def sd_set_temperature(self, tau: float):
        self._check(self._lib.sd_set_temperature(self._h, tau), "sd_set_temperature")

    def sd_set_verify_shape(self, shape: int):
        self._check(self._lib.sd_set_verify_shape(self._h, shape), "sd_set_verify_shape")

    def sd_set_active_count(self, count: Optional[torch.Tensor]):
        ptr = _dev(count, torch.int32, "count", allow_none=True)
        self._keep_count = count
        self._check(self._lib.sd_set_active_count(self._h, ptr), "sd_set_active_count")

    def sd_set_start_prediction(self, D_start: Optional[torch.Tensor]):
        ptr = _dev(D_start, torch.float32, "D_start", allow_none=True)
        self._keep_start = D_start
        self._check(self._lib.sd_set_start_prediction(self._h, ptr), "sd_set_start_prediction")

    def sd_set_draft_mirror(self, mirror: Optional[torch.Tensor]):
        """mirror: int16 tensor holding bf16 bit patterns, shape of Ytilde."""
        self._keep_mirror = mirror
        self._check(self._lib.sd_set_draft_mirror(self._h, _dev(mirror, torch.int16, "mirror", True)), "sd_set_draft_mirror")

    def sd_set_carry(self, Dq_ext: Optional[torch.Tensor], D_frozen: Optional[torch.Tensor]):
        self._keep_carry = (Dq_ext, D_frozen)
        self._check(self._lib.sd_set_carry(self._h, _dev(Dq_ext, torch.float32, "Dq_ext", True),
                                           _dev(D_frozen, torch.float32, "D_frozen", True)), "sd_set_carry")

    def sd_set_carry_rule(self, rule: int):
        self._check(self._lib.sd_set_carry_rule(self._h, int(rule)), "sd_set_carry_rule")

    def sd_workspace_bytes(self, Bmax: int) -> int:
        return int(self._lib.sd_workspace_bytes(self._h, Bmax))

    def sd_set_workspace(self, ws: Optional[torch.Tensor]):
        self._ws = ws
        if ws is None:
            self._check(self._lib.sd_set_workspace(self._h, None, 0), "sd_set_workspace")
        else:
            if not ws.is_cuda or not ws.is_contiguous():
                raise SDError("workspace: need a contiguous CUDA tensor")
            self._check(self._lib.sd_set_workspace(self._h, ws.data_ptr(), ws.numel() * ws.element_size()),
                        "sd_set_workspace")

    # -- window calls
    def sd_init_state(self, B, chain_id, y, n):
        self._check(self._lib.sd_init_state(self._h, B, _dev(chain_id, torch.int64, "chain_id"),
                                            _dev(y, torch.float32, "y"), _dev(n, torch.int32, "n"),
                                            _stream()), "sd_init_state")

    def sd_draft(self, B, y, n, chain_id, D0, Ytilde, krow):
        self._check(self._lib.sd_draft(self._h, B, _dev(y, torch.float32, "y"), _dev(n, torch.int32, "n"),
                                       _dev(chain_id, torch.int64, "chain_id"), _dev(D0, torch.float32, "D0"),
                                       _dev(Ytilde, torch.float32, "Ytilde"), _dev(krow, torch.int32, "krow"),
                                       _stream()), "sd_draft")

    def sd_draft_step(self, B, j, prev, n, chain_id, Dp, mp, Ytilde, krow, next=None, knext=None):
        self._check(self._lib.sd_draft_step(
            self._h, B, j, _dev(prev, torch.float32, "prev"), _dev(n, torch.int32, "n"),
            _dev(chain_id, torch.int64, "chain_id"), _dev(Dp, torch.float32, "Dp"),
            _dev(mp, torch.float32, "mp"), _dev(Ytilde, torch.float32, "Ytilde"),
            _dev(krow, torch.int32, "krow"), _dev(next, torch.float32, "next", True),
            _dev(knext, torch.int32, "knext", True), _stream()), "sd_draft_step")

    def sd_verify(self, B, y, n, chain_id, D0_or_mp, Dq, Ytilde, y_out, adv, rejected=None,
                  logratio=None, logu=None):
        self._check(self._lib.sd_verify(
            self._h, B, _dev(y, torch.float32, "y"), _dev(n, torch.int32, "n"),
            _dev(chain_id, torch.int64, "chain_id"), _dev(D0_or_mp, torch.float32, "D0_or_mp"),
            _dev(Dq, torch.float32, "Dq"), _dev(Ytilde, torch.float32, "Ytilde"),
            _dev(y_out, torch.float32, "y_out"), _dev(adv, torch.int32, "adv"),
            _dev(rejected, torch.uint8, "rejected", True), _dev(logratio, torch.float32, "logratio", True),
            _dev(logu, torch.float32, "logu", True), _stream()), "sd_verify")

    def sd_advance(self, B, y_out, adv, rejected, y, n, chain_id, out, B_active, counters=None):
        self._check(self._lib.sd_advance(
            self._h, B, _dev(y_out, torch.float32, "y_out"), _dev(adv, torch.int32, "adv"),
            _dev(rejected, torch.uint8, "rejected", True), _dev(y, torch.float32, "y"),
            _dev(n, torch.int32, "n"), _dev(chain_id, torch.int64, "chain_id"),
            _dev(out, torch.float32, "out"), _dev(B_active, torch.int32, "B_active"),
            _dev(counters, torch.int64, "counters", True), _stream()), "sd_advance")

    def sd_advance_static(self, B, y_out, adv, rejected, y, n, chain_id, out, B_active, counters=None):
        self._check(self._lib.sd_advance_static(
            self._h, B, _dev(y_out, torch.float32, "y_out"), _dev(adv, torch.int32, "adv"),
            _dev(rejected, torch.uint8, "rejected", True), _dev(y, torch.float32, "y"),
            _dev(n, torch.int32, "n"), _dev(chain_id, torch.int64, "chain_id"),
            _dev(out, torch.float32, "out"), _dev(B_active, torch.int32, "B_active"),
            _dev(counters, torch.int64, "counters", True), _stream()), "sd_advance_static")

    def sd_langevin_window(self, B, x, n, chain_id, means, logw, comp_std, M, gamma, x_out, adv,
                           rejected=None, logratio=None, logu=None):
        self._check(self._lib.sd_langevin_window(
            self._h, B, _dev(x, torch.float32, "x"), _dev(n, torch.int32, "n"),
            _dev(chain_id, torch.int64, "chain_id"), _dev(means, torch.float32, "means"),
            _dev(logw, torch.float32, "logw"), comp_std, M, gamma, _dev(x_out, torch.float32, "x_out"),
            _dev(adv, torch.int32, "adv"), _dev(rejected, torch.uint8, "rejected", True),
            _dev(logratio, torch.float32, "logratio", True), _dev(logu, torch.float32, "logu", True),
            _stream()), "sd_langevin_window")

    def sd_langevin_window_phi4(self, B, x, n, chain_id, L, beta, gamma, x_out, adv, rejected=None,
                                logratio=None, logu=None):
        self._check(self._lib.sd_langevin_window_phi4(
            self._h, B, _dev(x, torch.float32, "x"), _dev(n, torch.int32, "n"),
            _dev(chain_id, torch.int64, "chain_id"), L, beta, gamma, _dev(x_out, torch.float32, "x_out"),
            _dev(adv, torch.int32, "adv"), _dev(rejected, torch.uint8, "rejected", True),
            _dev(logratio, torch.float32, "logratio", True), _dev(logu, torch.float32, "logu", True),
            _stream()), "sd_langevin_window_phi4")

    def sd_langevin_run(self, B, x, n, chain_id, means, logw, comp_std, M, gamma, max_windows, x_out, n_out,
                        counters=None):
        self._check(self._lib.sd_langevin_run(
            self._h, B, _dev(x, torch.float32, "x"), _dev(n, torch.int32, "n"),
            _dev(chain_id, torch.int64, "chain_id"), _dev(means, torch.float32, "means"),
            _dev(logw, torch.float32, "logw"), comp_std, M, gamma, max_windows,
            _dev(x_out, torch.float32, "x_out"), _dev(n_out, torch.int32, "n_out"),
            _dev(counters, torch.int64, "counters", True), _stream()), "sd_langevin_run")

    def sd_langevin_chains(self, B, x, n, chain_id, means, logw, comp_std, M, gamma, out, B_active, counters=None) -> bool:
        """False when the chains have to be run window by window (nothing was enqueued then)."""
        rc = self._lib.sd_langevin_chains(
            self._h, B, _dev(x, torch.float32, "x"), _dev(n, torch.int32, "n"),
            _dev(chain_id, torch.int64, "chain_id"), _dev(means, torch.float32, "means"),
            _dev(logw, torch.float32, "logw"), comp_std, M, gamma, _dev(out, torch.float32, "out"),
            _dev(B_active, torch.int32, "B_active"), _dev(counters, torch.int64, "counters", True), _stream())
        if rc == SD_ERR_UNSUPPORTED:
            return False
        self._check(rc, "sd_langevin_chains")
        return True

    def sd_langevin_run_phi4(self, B, x, n, chain_id, L, beta, gamma, max_windows, x_out, n_out, counters=None):
        self._check(self._lib.sd_langevin_run_phi4(
            self._h, B, _dev(x, torch.float32, "x"), _dev(n, torch.int32, "n"),
            _dev(chain_id, torch.int64, "chain_id"), L, beta, gamma, max_windows,
            _dev(x_out, torch.float32, "x_out"), _dev(n_out, torch.int32, "n_out"),
            _dev(counters, torch.int64, "counters", True), _stream()), "sd_langevin_run_phi4")


class Denoiser:
    """Owns one ``sdden``; built by the ``sdden_*_create`` class methods."""

    def __init__(self, handle, d: int):
        self._lib = load_library()
        self._h = handle
        self.d = d

    @staticmethod
    def _created(rc, h, what):
        lib = load_library()
        if rc != 0:
            raise SDError(f"{what} failed ({rc}): {lib.sdden_last_error(None).decode()}")
        return h

    @classmethod
    def sdden_gmm_create(cls, means, stds, logw, alpha_bar_state):
        lib = load_library()
        mu, sd, lw, ab = (_host(v, np.float32) for v in (means, stds, logw, alpha_bar_state))
        M, d = mu.shape
        h = c_void_p()
        rc = lib.sdden_gmm_create(M, d, mu.ctypes.data, sd.ctypes.data, lw.ctypes.data, ab.shape[0] - 1,
                                  ab.ctypes.data, ctypes.byref(h))
        den = cls(cls._created(rc, h, "sdden_gmm_create"), d)
        den.components = M
        return den

    @classmethod
    def sdden_lowrank_create(cls, mu, U, s2, alpha_bar_state):
        lib = load_library()
        mu, U, ab = (_host(v, np.float32) for v in (mu, U, alpha_bar_state))
        d, r = U.shape
        h = c_void_p()
        rc = lib.sdden_lowrank_create(d, r, mu.ctypes.data, U.ctypes.data, float(s2), ab.shape[0] - 1,
                                      ab.ctypes.data, ctypes.byref(h))
        return cls(cls._created(rc, h, "sdden_lowrank_create"), d)

    @classmethod
    def sdden_mlp_create(cls, p, T: int, Rmax: int):
        lib = load_library()
        W1, W2, W3 = (_host(v, np.uint16) for v in (p.W1, p.W2, p.W3))
        b1, b2, b3 = (_host(v, np.float32) for v in (p.b1, p.b2, p.b3))
        h = c_void_p()
        rc = lib.sdden_mlp_create(p.d, p.H, p.E, W1.ctypes.data, b1.ctypes.data, W2.ctypes.data,
                                  b2.ctypes.data, W3.ctypes.data, b3.ctypes.data, T, Rmax, ctypes.byref(h))
        den = cls(cls._created(rc, h, "sdden_mlp_create"), p.d)
        den.wants_bf16 = True                      # first layer reads bf16: sdden_eval_mirror saves a conversion pass
        return den

    @classmethod
    def sdden_mlp4_create(cls, p, group: int, T: int, Rmax: int):
        """p: the bf16 network, as for ``sdden_mlp_create``; its matrices are quantised by the library."""
        lib = load_library()
        W1, W2, W3 = (_host(v, np.uint16) for v in (p.W1, p.W2, p.W3))
        b1, b2, b3 = (_host(v, np.float32) for v in (p.b1, p.b2, p.b3))
        if W1.shape != (p.d + p.E, p.H) or W2.shape != (p.H, p.H) or W3.shape != (p.H, p.d):
            raise SDError(f"sdden_mlp4_create: weights of shapes {W1.shape}, {W2.shape}, {W3.shape} do not fit d={p.d}, H={p.H}, E={p.E}")
        _check_group(group, "sdden_mlp4_create")
        h = c_void_p()
        rc = lib.sdden_mlp4_create(p.d, p.H, p.E, group, W1.ctypes.data, b1.ctypes.data, W2.ctypes.data, b2.ctypes.data,
                                   W3.ctypes.data, b3.ctypes.data, T, Rmax, ctypes.byref(h))
        den = cls(cls._created(rc, h, "sdden_mlp4_create"), p.d)
        den.wants_bf16 = True
        return den

    @classmethod
    def sdden_gated_create(cls, p, T: int, Rmax: int):
        """p: ``workloads.GatedParams`` (or the same fields)."""
        lib = load_library()
        We, Wg, Wu, Wd = (_host(v, np.uint16) for v in (p.We, p.Wg, p.Wu, p.Wd))
        be, nw, nb = (_host(v, np.float32) for v in (p.be, p.norm_weight, p.norm_bias))
        L, H, d = Wg.shape
        if Wu.shape != (L, H, d) or Wd.shape != (L, d, H) or nw.shape != (L, d) or nb.shape != (L, d) or be.shape != (d,) \
                or We.ndim != 2 or We.shape[1] != d:
            raise SDError("sdden_gated_create: the parameters' shapes do not fit each other")
        h = c_void_p()
        rc = lib.sdden_gated_create(d, H, We.shape[0], L, p.act, We.ctypes.data, be.ctypes.data, nw.ctypes.data, nb.ctypes.data, p.eps,
                                    Wg.ctypes.data, Wu.ctypes.data, Wd.ctypes.data, T, Rmax, ctypes.byref(h))
        return cls(cls._created(rc, h, "sdden_gated_create"), d)

    def _check(self, rc, what):
        if rc != 0:
            raise SDError(f"{what} failed ({rc}): {self._lib.sdden_last_error(self._h).decode()}")

    def sdden_eval(self, R, X, krow, out):
        """X, out may be views into larger buffers (their first element is what is passed)."""
        rc = self._lib.sdden_eval(self._h, R, _dev(X, torch.float32, "X"), _dev(krow, torch.int32, "krow"),
                                  _dev(out, torch.float32, "out"), _stream())
        if rc != 0:
            self._check(rc, "sdden_eval")

    def sdden_eval_mirror(self, R, X, Xbf16, krow, out):
        rc = self._lib.sdden_eval_mirror(self._h, R, _dev(X, torch.float32, "X"), _dev(Xbf16, torch.int16, "Xbf16"),
                                         _dev(krow, torch.int32, "krow"), _dev(out, torch.float32, "out"), _stream())
        if rc != 0:
            self._check(rc, "sdden_eval_mirror")

    def sdden_run(self, ctx: Context, B, y, n, chain_id, out, B_active, counters=None, D_frozen=None, draft_den=None) -> bool:
        """False when the chains of this denoiser have to be run window by window (nothing was enqueued then)."""
        rc = self._lib.sdden_run(self._h, draft_den._h if draft_den is not None else None, ctx._h, B, _dev(y, torch.float32, "y"),
                                 _dev(n, torch.int32, "n"), _dev(chain_id, torch.int64, "chain_id"),
                                 _dev(D_frozen, torch.float32, "D_frozen", True), _dev(out, torch.float32, "out"),
                                 _dev(B_active, torch.int32, "B_active"), _dev(counters, torch.int64, "counters", True), _stream())
        if rc == SD_ERR_UNSUPPORTED:
            return False
        self._check(rc, "sdden_run")
        return True

    def sdden_reserve(self, Rmax: int):
        self._check(self._lib.sdden_reserve(self._h, Rmax), "sdden_reserve")

    def sdden_profile(self, which: int):
        self._check(self._lib.sdden_profile(self._h, which), "sdden_profile")

    def sdden_profile_min_rows(self, min_rows: int):
        self._check(self._lib.sdden_profile_min_rows(self._h, min_rows), "sdden_profile_min_rows")

    def sdden_profile_collect(self):
        ms, n = ctypes.c_double(), c_int64()
        self._check(self._lib.sdden_profile_collect(self._h, ctypes.byref(ms), ctypes.byref(n)),
                    "sdden_profile_collect")
        return ms.value, n.value

    def sdden_mlp_select_gemm(self, variant: int):
        self._check(self._lib.sdden_mlp_select_gemm(self._h, variant), "sdden_mlp_select_gemm")

    def sdden_set_active_count(self, count: Optional[torch.Tensor], rows_per_chain: int = 1):
        self._keep_count = count
        ptr = _dev(count, torch.int32, "count", allow_none=True)
        self._check(self._lib.sdden_set_active_count(self._h, ptr, rows_per_chain), "sdden_set_active_count")

    def close(self):
        if getattr(self, "_h", None):
            self._lib.sdden_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


# -- layers of row networks: functions of tensors on the current device, on its current stream.  Calls on few rows are bound by
# the host, so the checks ask each tensor once and build their messages only when one fails.
_F32, _BF16 = torch.float32, torch.bfloat16
_LAYER_TYPES = {_F32: SDDEN_F32, _BF16: SDDEN_BF16}
_MAX_ROWS = 1 << 30


def _rows(t: Optional[torch.Tensor], name: str, shape=None, only=None, allow_none: bool = False):
    """(pointer, stride between rows) of an fp32 or bf16 matrix (or of type ``only``) whose rows are contiguous and need not follow
    each other."""
    if t is None:
        if allow_none:
            return None, 0
        raise SDError(f"{name}: tensor required")
    dims, dtype = t.shape, t.dtype
    if not t.is_cuda or t.get_device() != torch._C._cuda_getDevice() or len(dims) != 2 or (dtype is not only if only is not None else dtype not in _LAYER_TYPES):
        raise SDError(f"{name}: need a matrix of {only or 'fp32 or bf16'} on the current device, got {dtype} {tuple(dims)} on {t.device}")
    if shape is not None and dims != shape:
        raise SDError(f"{name}: need shape {tuple(shape)}, got {tuple(dims)}")
    R, d = dims
    if R > _MAX_ROWS or d > _MAX_ROWS:               # the library's sizes are 32 bits wide
        raise SDError(f"{name}: {R} rows of {d} are more than one call takes (2^30)")
    stride, inner = t.stride()
    if inner != 1 and d > 1:
        raise SDError(f"{name}: the elements of a row must be contiguous, got strides {t.stride()}")
    if R <= 1:
        stride = d if d > 0 else 1
    elif stride < d:
        raise SDError(f"{name}: rows overlap (stride {stride} of {d} columns)")
    return t.data_ptr(), stride


def _flat(t: Optional[torch.Tensor], name: str, shape, dtype, allow_none: bool = False) -> Optional[int]:
    """Pointer of a contiguous tensor of this shape and type on the current device."""
    if t is None:
        if allow_none:
            return None
        raise SDError(f"{name}: tensor required")
    if t.dtype is dtype and t.shape == shape and t.is_contiguous() and t.is_cuda and t.get_device() == torch._C._cuda_getDevice():
        return t.data_ptr()
    raise SDError(f"{name}: need a contiguous {dtype} tensor of shape {tuple(shape)} on the current device, got {t.dtype} "
                  f"{tuple(t.shape)} on {t.device}, contiguous={t.is_contiguous()}")


def _hidden_width(Wg) -> int:
    """H of the gate weights [H,d], from which the other shapes follow."""
    if Wg is None or len(Wg.shape) != 2:
        raise SDError(f"Wg: need a matrix [H,d], got {None if Wg is None else tuple(Wg.shape)}")
    return Wg.shape[0]


def _scratch(t: Optional[torch.Tensor], name: str):
    """(pointer, bytes) of a caller's workspace, any contiguous tensor."""
    if t is None:
        return None, 0
    if not t.is_cuda or t.get_device() != torch._C._cuda_getDevice() or not t.is_contiguous():
        raise SDError(f"{name}: need a contiguous tensor on the current device")
    return t.data_ptr(), t.numel() * t.element_size()


def _layer_check(lib, rc: int, what: str):
    if rc != 0:
        raise SDError(f"{what} failed ({rc}): {lib.sdden_last_error(None).decode()}")


def _check_group(group: int, what: str):
    """ctypes would hand on the low 32 bits of a larger number: another group than the scales were laid out for."""
    if not 0 < group < 1 << 31:
        raise SDError(f"{what}: group={group} must be positive and below 2^31")


def sdden_layernorm_workspace_bytes(R: int, d: int) -> int:
    return int(load_library().sdden_layernorm_workspace_bytes(R, d))


def sdden_layernorm_forward(x, weight, bias, eps: float, y, mean=None, rstd=None):
    """x, y [R,d] fp32 or bf16, rows may lie apart; weight, bias [d] fp32 or None; mean, rstd [R] fp32 or both None."""
    lib = load_library()
    xp, xs = _rows(x, "x")
    R, d = x.shape
    yp, ys = _rows(y, "y", (R, d))
    _layer_check(lib, lib.sdden_layernorm_forward(
        R, d, xp, _LAYER_TYPES[x.dtype], xs, _flat(weight, "weight", (d,), torch.float32, True),
        _flat(bias, "bias", (d,), torch.float32, True), eps, yp, _LAYER_TYPES[y.dtype], ys,
        _flat(mean, "mean", (R,), torch.float32, True), _flat(rstd, "rstd", (R,), torch.float32, True), _stream()),
        "sdden_layernorm_forward")


def sdden_layernorm_backward(dy, x, weight, mean, rstd, dx, dweight=None, dbias=None, workspace=None, dres=None):
    """dres and dx have x's type; dweight, dbias [d] fp32 or None; workspace: any tensor of sdden_layernorm_workspace_bytes."""
    lib = load_library()
    xp, xs = _rows(x, "x")
    R, d = x.shape
    dyp, dys = _rows(dy, "dy", (R, d))
    dxp, dxs = _rows(dx, "dx", (R, d), x.dtype)
    drp, drs = _rows(dres, "dres", (R, d), x.dtype, True)
    ws, nbytes = _scratch(workspace, "workspace")
    _layer_check(lib, lib.sdden_layernorm_backward(
        R, d, dyp, _LAYER_TYPES[dy.dtype], dys, xp, _LAYER_TYPES[x.dtype], xs, _flat(weight, "weight", (d,), torch.float32, True),
        _flat(mean, "mean", (R,), torch.float32), _flat(rstd, "rstd", (R,), torch.float32), drp, drs, dxp, dxs,
        _flat(dweight, "dweight", (d,), torch.float32, True), _flat(dbias, "dbias", (d,), torch.float32, True), ws, nbytes, _stream()),
        "sdden_layernorm_backward")


def sdden_gated_workspace_bytes(R: int, d: int, H: int) -> int:
    return int(load_library().sdden_gated_workspace_bytes(R, d, H))


def sdden_gated_forward(X, Wg, Wu, Wd, Y, hidden, gates=None, act: int = SDDEN_SILU, res=None):
    """X [R,d], Wg, Wu [H,d], Wd [d,H], hidden [R,H] bf16; Y and res [R,d] fp32 or bf16; gates [2,R,H] fp32 or None."""
    lib = load_library()
    bf = _BF16
    xp, xs = _rows(X, "X", only=bf)
    R, d = X.shape
    H = _hidden_width(Wg)
    yp, ys = _rows(Y, "Y", (R, d))
    rp, rs = _rows(res, "res", (R, d), Y.dtype, True)
    if res is not None and R > 1 and rs != ys:
        raise SDError(f"res: its rows must lie as far apart as Y's ({ys}), got {rs}")
    _layer_check(lib, lib.sdden_gated_forward(
        R, d, H, act, xp, xs, _flat(Wg, "Wg", (H, d), bf), _flat(Wu, "Wu", (H, d), bf), _flat(Wd, "Wd", (d, H), bf), rp, yp,
        _LAYER_TYPES[Y.dtype], ys, _flat(hidden, "hidden", (R, H), bf), _flat(gates, "gates", (2, R, H), torch.float32, True), _stream()),
        "sdden_gated_forward")


def sdden_gated_backward(dY, X, Wg, Wu, Wd, gates, hidden, dX, dWg, dWu, dWd, workspace, act: int = SDDEN_SILU):
    """dX [R,d] bf16 or None; dWg, dWu [H,d], dWd [d,H] fp32 or bf16, or all None; workspace: any tensor of
    sdden_gated_workspace_bytes."""
    lib = load_library()
    bf = _BF16
    xp, xs = _rows(X, "X", only=bf)
    R, d = X.shape
    H = _hidden_width(Wg)
    dyp, dys = _rows(dY, "dY", (R, d), bf)
    dxp, dxs = _rows(dX, "dX", (R, d), bf, True)
    tw = torch.float32 if dWg is None else dWg.dtype
    if tw not in _LAYER_TYPES:
        raise SDError(f"dWg: need fp32 or bf16, got {tw}")
    ws, nbytes = _scratch(workspace, "workspace")
    _layer_check(lib, lib.sdden_gated_backward(
        R, d, H, act, dyp, dys, xp, xs, _flat(Wg, "Wg", (H, d), bf), _flat(Wu, "Wu", (H, d), bf), _flat(Wd, "Wd", (d, H), bf),
        _flat(gates, "gates", (2, R, H), torch.float32), _flat(hidden, "hidden", (R, H), bf), dxp, dxs,
        _flat(dWg, "dWg", (H, d), tw, True), _flat(dWu, "dWu", (H, d), tw, True), _flat(dWd, "dWd", (d, H), tw, True),
        _LAYER_TYPES[tw], ws, nbytes, _stream()), "sdden_gated_backward")


class Q4Matrix:
    """Owns one ``sdden_q4``: a matrix in 4 bits on the device that was current when it was created."""

    def __init__(self, handle, N: int, K: int):
        self._lib = load_library()
        self._h = handle
        self.N, self.K = N, K

    @classmethod
    def sdden_q4_create(cls, q, scale, K: int, group: int):
        """q: uint8 [N, ceil(K/2)], two inputs per byte (the even one in the low half); scale: bf16 bit patterns, uint16 (or the
        same as int16) [N, ceil(K/group)]."""
        lib = load_library()
        q, scale = np.ascontiguousarray(q), np.ascontiguousarray(scale)
        if q.dtype != np.uint8 or scale.dtype not in (np.uint16, np.int16) or K <= 0 or group <= 0 or q.ndim != 2 \
                or q.shape[1] != (K + 1) // 2 or scale.shape != (q.shape[0], -(-K // group)):
            raise SDError(f"sdden_q4_create: need uint8 [N, ceil(K/2)] and 16-bit [N, ceil(K/group)] for K={K}, group={group}, got "
                          f"{q.dtype} {q.shape} and {scale.dtype} {scale.shape}")
        _check_group(group, "sdden_q4_create")
        h = c_void_p()
        rc = lib.sdden_q4_create(q.shape[0], K, group, q.ctypes.data, scale.ctypes.data, ctypes.byref(h))
        _layer_check(lib, rc, "sdden_q4_create")
        return cls(h, q.shape[0], K)

    def sdden_q4_eval(self, X, Y, bias=None):
        """X [R,K], Y [R,N] fp32 or bf16, rows may lie apart; bias [N] fp32 or None."""
        xp, xs = _rows(X, "X")
        if X.shape[1] != self.K:
            raise SDError(f"X: need {self.K} columns, got {X.shape[1]}")
        yp, ys = _rows(Y, "Y", (X.shape[0], self.N))
        rc = self._lib.sdden_q4_eval(self._h, X.shape[0], xp, _LAYER_TYPES[X.dtype], xs, _flat(bias, "bias", (self.N,), torch.float32, True),
                                     yp, _LAYER_TYPES[Y.dtype], ys, _stream())
        if rc != 0:
            _layer_check(self._lib, rc, "sdden_q4_eval")

    def close(self):
        if getattr(self, "_h", None):
            self._lib.sdden_q4_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def sd_measure_stream(src: Optional[torch.Tensor], dst: torch.Tensor, nbytes: int, mode: int, workgroups: int = 0):
    """Measurement kernel (include/sd_measure.h): streaming copy (0), read (1) or fill (2) of nbytes; 3, 4, 5 the
    same with a workgroup walking whole 48 KiB rows."""
    lib = load_library()
    rc = lib.sd_measure_stream(None if src is None else src.data_ptr(), dst.data_ptr(), nbytes, mode, workgroups, _stream())
    if rc != 0:
        raise SDError(f"sd_measure_stream failed ({rc})")


def sd_measure_mfma(shape: int, iters: int, sink: torch.Tensor, workgroups: int = 0) -> float:
    """Measurement kernel (include/sd_measure.h): a loop of MFMAs on register operands; returns its flops."""
    lib = load_library()
    fl = ctypes.c_double()
    rc = lib.sd_measure_mfma(shape, iters, workgroups, sink.data_ptr(), ctypes.byref(fl), _stream())
    if rc != 0:
        raise SDError(f"sd_measure_mfma failed ({rc})")
    return fl.value
