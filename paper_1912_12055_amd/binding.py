"""Thin ctypes binding of the C ABI in include/nna.h.

Argument marshalling only: every step of the transforms runs in the HIP library.
PyTorch supplies device memory and streams.  There is no fallback: if libnna.so is
missing the import of this module's functions raises.
"""
from __future__ import annotations

import array
import ctypes
import operator
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libnna.so")

NNA_OK = 0
NNA_ERR_INVALID_ARG, NNA_ERR_UNSUPPORTED, NNA_ERR_SHAPE, NNA_ERR_ALLOC, NNA_ERR_HIP = 1, 2, 3, 4, 5
NNA_OUT_MAGNITUDE, NNA_OUT_POWER, NNA_OUT_LOG, NNA_OUT_COMPLEX, NNA_OUT_PHASE = 0, 1, 2, 3, 4
NNA_WIN_HANN, NNA_WIN_RECT, NNA_WIN_HAMMING, NNA_WIN_BLACKMAN = 0, 1, 2, 3
NNA_MEL_SLANEY, NNA_MEL_HTK = 0, 1
NNA_FREQ_LINEAR, NNA_FREQ_LOG = 1, 2
NNA_PREC_F32, NNA_PREC_F16 = 0, 1
NNA_KIND_STFT, NNA_KIND_MEL, NNA_KIND_CQT, NNA_KIND_CQT2010V2, NNA_KIND_CQT1992, NNA_KIND_CQT2010 = 0, 1, 2, 3, 4, 5

# every symbol include/nna.h declares
EXPORTS = [
    "nna_plan_stft", "nna_plan_stft_prec", "nna_plan_stft_scaled", "nna_plan_mel", "nna_plan_cqt", "nna_plan_cqt2010v2", "nna_out_shape", "nna_stft", "nna_mel", "nna_cqt",
    "nna_plan_bank", "nna_plan_mel_weights", "nna_plan_info", "nna_plan_cqt_lengths", "nna_plan_sigma", "nna_cqt2010v2_workspace",
    "nna_cqt2010v2", "nna_plan_part", "nna_plan_cqt1992", "nna_cqt1992", "nna_plan_spectral_kernels",
    "nna_plan_cqt2010", "nna_cqt2010",
    "nna_plan_get_mel_weights", "nna_plan_set_mel_weights", "nna_mel_backward_workspace", "nna_mel_backward",
    "nna_plan_trainable", "nna_plan_get_bank", "nna_plan_set_bank", "nna_stft_backward_workspace", "nna_stft_backward",
    "nna_cqt_backward_workspace", "nna_cqt_backward", "nna_mel_with_stft", "nna_cqt2010v2_static",
    "nna_cqt2010v2_backward_workspace", "nna_cqt2010v2_backward",
    "nna_plan_get_spectral_kernels", "nna_plan_set_spectral_kernels", "nna_cqt1992_backward_workspace", "nna_cqt1992_backward",
    "nna_cqt2010_backward_workspace", "nna_cqt2010_backward", "nna_kept_bytes", "nna_forward_keep", "nna_backward_kept", "nna_plan_applied_kernels", "nna_plan_applied_tiles", "nna_plan_short_tiles",
    "nna_plan_destroy",
    "nna_status_str", "nna_last_error",
    "nna_cqt_workspace", "nna_cqt_in_workspace",
    "nna_layer_norm", "nna_layer_norm_frames", "nna_layer_norm_backward_workspace", "nna_layer_norm_backward",
    "nna_layer_norm_frames_backward", "nna_pack8", "nna_unpack8",
    "nna_decay_attention_workspace", "nna_decay_attention_backward_workspace", "nna_decay_attention", "nna_decay_attention_backward", "nna_decay_attention_step",
    "nna_rotate_heads", "nna_rotate_heads_backward_workspace", "nna_rotate_heads_backward",
    "nna_gated_scan_workspace", "nna_gated_scan", "nna_gated_scan_backward", "nna_gated_scan_step",
    "nna_adamw", "nna_adamw_steps", "nna_adamw_moment",
]

_c = ctypes
_LL = _c.c_longlong
_VP = _c.c_void_p
_lib = None


class NnaError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"nna status {status}: {message}")
        self.status = status
        self.message = message


def lib():
    """Load libnna.so (built in-tree by build.py / __graft_entry__.build())."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_1912_12055_amd.build` "
                "(there is no CPU fallback)")
        # PyTorch ships a HIP runtime of its own.  Loading it first makes the library's dependency on
        # the runtime resolve to that copy, so the process holds one runtime; loaded the other way
        # round, the second copy finds no device.
        try:
            import torch  # noqa: F401
        except ImportError:
            pass
        L = _c.CDLL(LIB_PATH)
        PP = _c.POINTER(_VP)
        L.nna_plan_stft.argtypes = [PP, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int]
        L.nna_plan_stft_prec.argtypes = [PP, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                         _c.c_int]
        L.nna_plan_stft_scaled.argtypes = [PP, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                           _c.c_double, _c.c_double, _c.c_int, _c.c_int]
        L.nna_plan_mel.argtypes = [PP, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_double,
                                   _c.c_double, _c.c_int, _c.c_int, _c.c_double, _c.c_int]
        L.nna_plan_cqt.argtypes = [PP, _c.c_int, _c.c_int, _c.c_double, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                   _c.c_int, _c.c_int, _c.c_int]
        L.nna_plan_cqt2010v2.argtypes = [PP, _c.c_int, _c.c_int, _c.c_double, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                         _c.c_int, _c.c_int, _c.c_int]
        L.nna_plan_cqt1992.argtypes = [PP, _c.c_int, _c.c_int, _c.c_double, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                       _c.c_int, _c.c_int, _c.c_int]
        L.nna_plan_spectral_kernels.argtypes = [_VP, _c.POINTER(_c.c_double), _c.c_size_t]
        L.nna_cqt2010v2_workspace.argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_cqt_workspace.argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_cqt_in_workspace.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _c.c_size_t, _VP]
        L.nna_cqt2010v2.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _c.c_size_t, _VP]
        L.nna_cqt2010.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _c.c_size_t, _VP]
        L.nna_plan_cqt2010.argtypes = [PP, _c.c_int, _c.c_int, _c.c_double, _c.c_int, _c.c_int, _c.c_int, _c.c_int,
                                       _c.c_int, _c.c_int, _c.c_int]
        L.nna_plan_part.argtypes = [_VP, _c.c_int, PP]
        L.nna_plan_get_mel_weights.argtypes = [_VP, _VP, _VP]
        L.nna_plan_set_mel_weights.argtypes = [_VP, _VP, _VP]
        L.nna_mel_backward_workspace.argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_mel_backward.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _VP]
        L.nna_plan_trainable.argtypes = [_VP]
        L.nna_plan_get_bank.argtypes = [_VP, _VP, _VP]
        L.nna_plan_set_bank.argtypes = [_VP, _VP, _VP]
        L.nna_stft_backward_workspace.argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_stft_backward.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _VP, _VP, _c.c_size_t, _VP]
        L.nna_cqt_backward_workspace.argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_cqt_backward.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _VP, _VP, _c.c_size_t, _VP]
        L.nna_kept_bytes.argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_forward_keep.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _VP, _c.c_size_t, _VP]
        L.nna_backward_kept.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _c.c_size_t, _VP, _VP, _VP, _VP, _c.c_size_t, _VP]
        L.nna_cqt2010v2_backward_workspace.argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_cqt2010v2_backward.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _VP, _VP, _c.c_size_t, _VP]
        L.nna_plan_get_spectral_kernels.argtypes = [_VP, _VP, _VP]
        L.nna_plan_set_spectral_kernels.argtypes = [_VP, _VP, _VP]
        for name in ("nna_cqt1992", "nna_cqt2010"):
            getattr(L, name + "_backward_workspace").argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_size_t)]
            getattr(L, name + "_backward").argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _VP]
        L.nna_mel_with_stft.argtypes = [_VP, _VP, _LL, _LL, _VP, _VP, _VP]
        _I, _D = _c.c_int, _c.c_double
        L.nna_layer_norm.argtypes = [_VP, _I, _LL, _LL, _LL, _VP, _VP, _D, _VP, _I, _VP, _VP, _VP, _I, _VP]
        L.nna_layer_norm_frames.argtypes = [_VP, _LL, _LL, _LL, _VP, _VP, _D, _VP, _I, _VP, _I, _VP]
        L.nna_layer_norm_backward_workspace.argtypes = [_LL, _LL, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_layer_norm_backward.argtypes = [_VP, _I, _VP, _I, _LL, _LL, _LL, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _I, _VP]
        L.nna_layer_norm_frames_backward.argtypes = [_VP, _I, _VP, _LL, _LL, _LL, _VP, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _I, _VP]
        L.nna_pack8.argtypes = [_VP, _I, _LL, _LL, _LL, _VP, _VP, _I, _VP]
        L.nna_unpack8.argtypes = [_VP, _VP, _LL, _LL, _VP, _I, _I, _VP]
        qkv, shape = 3 * [_VP, _c.POINTER(_LL)], 5 * [_LL]
        L.nna_decay_attention_workspace.argtypes = L.nna_decay_attention_backward_workspace.argtypes = [*shape, _c.POINTER(_c.c_size_t)]
        L.nna_decay_attention.argtypes = [*qkv, _I, *shape, _VP, _D, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _I, _VP]
        L.nna_decay_attention_backward.argtypes = [_VP, *qkv, _I, *shape, _VP, _D, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _I, _VP]
        L.nna_decay_attention_step.argtypes = [*qkv, _I, _LL, _LL, _LL, _LL, _VP, _D, _VP, _VP, _I, _VP]
        _PLL = _c.POINTER(_LL)
        heads, turns = 2 * [_VP, _PLL, _LL] + [_I, _LL, _LL, _LL], [_VP, _LL, _I, _VP, _PLL, _LL, _I, _D, _VP, _VP]
        L.nna_rotate_heads.argtypes = [*heads, *turns, _VP, _VP, _I, _VP]
        L.nna_rotate_heads_backward_workspace.argtypes = [_LL, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_rotate_heads_backward.argtypes = [_VP, _VP, *heads, *turns, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _I, _VP]
        gates, frames = 3 * [_VP, _PLL], [_I, _LL, _LL, _LL, _VP]
        L.nna_gated_scan_workspace.argtypes = [_LL, _LL, _LL, _c.POINTER(_c.c_size_t)]
        L.nna_gated_scan.argtypes = [*gates, *frames, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _I, _VP]
        L.nna_gated_scan_backward.argtypes = [_VP, _VP, *gates, *frames, _VP, _VP, _VP, _VP, _VP, _VP, _c.c_size_t, _I, _VP]
        L.nna_gated_scan_step.argtypes = [_VP, _LL, _VP, _LL, _VP, _LL, _I, _LL, _LL, _VP, _VP, _I, _VP]
        L.nna_adamw.argtypes = [_VP, _VP, _VP, _VP, _LL, _VP, _VP, _VP, _VP, _VP, _LL, _LL, _VP, _D, _VP, _D, _D, _D, _D, _I, _VP]
        L.nna_adamw_steps.argtypes = [_VP, _VP, _VP, _VP, _LL, _VP, _VP, _VP, _VP, _VP, _LL, _VP, _VP, _I, _D, _VP, _D, _D, _D, _D, _I, _VP]
        L.nna_adamw_moment.argtypes = [_VP, _I, _VP, _LL, _VP, _I, _VP]
        L.nna_out_shape.argtypes = [_VP, _LL, _LL, _c.POINTER(_LL), _c.POINTER(_LL)]
        for name in ("nna_stft", "nna_mel", "nna_cqt", "nna_cqt1992", "nna_cqt2010v2_static"):
            getattr(L, name).argtypes = [_VP, _VP, _LL, _LL, _VP, _VP]
        L.nna_plan_bank.argtypes = [_VP, _c.POINTER(_c.c_double), _c.c_size_t]
        L.nna_plan_applied_kernels.argtypes = [_VP, _c.POINTER(_c.c_double), _c.c_size_t, _c.POINTER(_LL)]
        L.nna_plan_applied_tiles.argtypes = [_VP, _LL, _LL, _c.POINTER(_c.c_int), _c.POINTER(_c.c_int)]
        L.nna_plan_short_tiles.argtypes = [_VP, _LL, _LL] + 4 * [_c.POINTER(_c.c_int)]
        L.nna_plan_mel_weights.argtypes = [_VP, _c.POINTER(_c.c_double), _c.c_size_t]
        L.nna_plan_info.argtypes = [_VP, _c.POINTER(_c.c_int), _c.POINTER(_LL), _c.POINTER(_LL), _c.POINTER(_LL),
                                    _c.POINTER(_c.c_double), _c.POINTER(_c.c_double)]
        L.nna_plan_cqt_lengths.argtypes = [_VP, _c.POINTER(_LL), _c.c_size_t]
        L.nna_plan_sigma.argtypes = [_VP, _c.POINTER(_c.c_double), _c.c_size_t]
        L.nna_plan_destroy.argtypes = [_VP]
        L.nna_plan_destroy.restype = None
        L.nna_status_str.argtypes = [_c.c_int]
        L.nna_status_str.restype = _c.c_char_p
        L.nna_last_error.restype = _c.c_char_p
        for name in EXPORTS:
            if name not in ("nna_plan_destroy", "nna_status_str", "nna_last_error"):
                getattr(L, name).restype = _c.c_int
        _lib = L
    return _lib


def nna_last_error() -> str:
    return lib().nna_last_error().decode()


def nna_status_str(status: int) -> str:
    return lib().nna_status_str(status).decode()


def _check(status: int):
    if status != NNA_OK:
        raise NnaError(status, nna_last_error() or nna_status_str(status))


class Plan:
    """Owns one nna_plan*; destroyed with the object."""

    def __init__(self, handle: int, device: int, owner=None):
        self.handle = handle
        self.device = device
        self.owner = owner  # a part of another plan: that plan owns the handle (and is kept alive here)
        self.bank_sets = 0  # calls of nna_plan_set_bank
        self._constants = None

    def __del__(self):
        h, self.handle = getattr(self, "handle", None), None
        if h and _lib is not None and getattr(self, "owner", None) is None:
            _lib.nna_plan_destroy(h)

    def info(self) -> dict:
        kind = _c.c_int()
        rows, taps, bins = _LL(), _LL(), _LL()
        ex, alg = _c.c_double(), _c.c_double()
        _check(lib().nna_plan_info(self.handle, kind, rows, taps, bins, ex, alg))
        return dict(kind=kind.value, bank_rows=rows.value, taps=taps.value, out_bins=bins.value,
                    executed_flops_per_frame=ex.value, algorithmic_flops_per_frame=alg.value)


    def constants(self):
        """(kind, bank rows, taps): asked for once, a plan never changes them."""
        if self._constants is None:
            i = self.info()
            self._constants = (i["kind"], i["bank_rows"], i["taps"])
        return self._constants


def _new_plan(fn, args, device):
    h = _VP()
    _check(fn(_c.byref(h), *args, device))
    return Plan(h.value, device)


def nna_plan_stft(sr=22050, n_fft=2048, hop=512, win=NNA_WIN_HANN, center=True, fmt=NNA_OUT_MAGNITUDE,
                  device=0) -> Plan:
    return _new_plan(lib().nna_plan_stft, (sr, n_fft, hop, win, int(center), fmt), device)


def nna_plan_stft_prec(sr=22050, n_fft=2048, hop=512, win=NNA_WIN_HANN, center=True, fmt=NNA_OUT_MAGNITUDE,
                       precision=NNA_PREC_F16, device=0) -> Plan:
    return _new_plan(lib().nna_plan_stft_prec, (sr, n_fft, hop, win, int(center), fmt, precision), device)


def nna_plan_stft_scaled(sr=22050, n_fft=2048, hop=512, win=NNA_WIN_HANN, center=True, fmt=NNA_OUT_MAGNITUDE,
                         freq_scale=NNA_FREQ_LINEAR, fmin=50.0, fmax=6000.0, freq_bins=0, device=0) -> Plan:
    return _new_plan(lib().nna_plan_stft_scaled,
                     (sr, n_fft, hop, win, int(center), fmt, freq_scale, float(fmin), float(fmax), freq_bins), device)


def nna_plan_mel(sr=22050, n_fft=2048, hop=512, win=NNA_WIN_HANN, center=True, n_mels=128, fmin=0.0, fmax=0.0,
                 scale=NNA_MEL_SLANEY, norm_area=True, power=2.0, device=0) -> Plan:
    return _new_plan(lib().nna_plan_mel,
                     (sr, n_fft, hop, win, int(center), n_mels, float(fmin), float(fmax), scale, int(norm_area),
                      float(power)), device)


def nna_plan_cqt(sr=22050, hop=512, fmin=32.70, n_bins=84, bins_per_octave=12, win=NNA_WIN_HANN, center=True,
                 n_taps=0, fmt=NNA_OUT_MAGNITUDE, device=0) -> Plan:
    return _new_plan(lib().nna_plan_cqt,
                     (sr, hop, float(fmin), n_bins, bins_per_octave, win, int(center), n_taps, fmt), device)


def nna_plan_cqt2010v2(sr=22050, hop=512, fmin=32.70, n_bins=84, bins_per_octave=12, win=NNA_WIN_HANN, n_taps=0,
                       fir_taps=0, fmt=NNA_OUT_MAGNITUDE, device=0) -> Plan:
    return _new_plan(lib().nna_plan_cqt2010v2,
                     (sr, hop, float(fmin), n_bins, bins_per_octave, win, n_taps, fir_taps, fmt), device)


def nna_plan_cqt1992(sr=22050, hop=512, fmin=32.70, n_bins=84, bins_per_octave=12, win=NNA_WIN_HANN, center=True,
                     n_fft=0, fmt=NNA_OUT_MAGNITUDE, device=0) -> Plan:
    plan = _new_plan(lib().nna_plan_cqt1992,
                     (sr, hop, float(fmin), n_bins, bins_per_octave, win, int(center), n_fft, fmt), device)
    plan.spectral_rows = 2 * n_bins  # rows of the spectral kernels as a tensor: (Re, Im) per constant-Q bin
    return plan


def nna_plan_spectral_kernels(plan: Plan) -> np.ndarray:
    """Complex [n_bins, n_fft/2+1]: the spectral kernels of a plan from nna_plan_cqt1992, divided by n_fft."""
    i = plan.info()
    # (a complex-format plan reports two output rows per bin; the constructor wrapper recorded the real count)
    out = np.empty((getattr(plan, "spectral_rows", 2 * i["out_bins"]), i["taps"] // 2 + 1), dtype=np.float64)
    _check(lib().nna_plan_spectral_kernels(plan.handle, out.ctypes.data_as(_c.POINTER(_c.c_double)), out.size))
    return out[0::2] + 1j * out[1::2]


def nna_plan_cqt2010(sr=22050, hop=512, fmin=32.70, n_bins=84, bins_per_octave=12, win=NNA_WIN_HANN, n_fft=0,
                     fir_taps=0, fmt=NNA_OUT_MAGNITUDE, device=0) -> Plan:
    plan = _new_plan(lib().nna_plan_cqt2010,
                     (sr, hop, float(fmin), n_bins, bins_per_octave, win, n_fft, fir_taps, fmt), device)
    plan.spectral_rows = 2 * min(n_bins, bins_per_octave)  # the top octave's kernels serve every octave
    return plan


def nna_plan_part(plan: Plan, index: int) -> Plan:
    """Octave `index` (0 = top) of a downsampling CQT plan, or its filter bank for index -1."""
    h = _VP()
    _check(lib().nna_plan_part(plan.handle, index, _c.byref(h)))
    return Plan(h.value, plan.device, owner=plan)


def nna_cqt2010v2_workspace(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_cqt2010v2_workspace(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_out_shape(plan: Plan, B: int, L: int):
    nb, nf = _LL(), _LL()
    _check(lib().nna_out_shape(plan.handle, B, L, nb, nf))
    return nb.value, nf.value


def nna_plan_bank(plan: Plan) -> np.ndarray:
    i = plan.info()
    out = np.empty((i["bank_rows"], i["taps"]), dtype=np.float64)
    _check(lib().nna_plan_bank(plan.handle, out.ctypes.data_as(_c.POINTER(_c.c_double)), out.size))
    return out


def nna_plan_applied_kernels(plan: Plan) -> np.ndarray:
    """The kernels a fixed constant-Q plan applies, [2 n_bins, K], multiplied out in 64 bits."""
    rows = _LL()
    _check(lib().nna_plan_applied_kernels(plan.handle, None, 0, _c.byref(rows)))
    out = np.empty((rows.value, plan.info()["taps"]), dtype=np.float64)
    _check(lib().nna_plan_applied_kernels(plan.handle, out.ctypes.data_as(_c.POINTER(_c.c_double)), out.size, None))
    return out


def nna_plan_applied_tiles(plan: Plan, B: int, L: int):
    """((frames, 16-frame blocks per wave) of the bins with a basis, the same of those taken tap by tap)."""
    f, b = (_c.c_int * 2)(), (_c.c_int * 2)()
    _check(lib().nna_plan_applied_tiles(plan.handle, B, L, f, b))
    return (f[0], b[0]), (f[1], b[1])


def nna_plan_short_tiles(plan: Plan, B: int, L: int):
    """(form, frames per tile, columns at a time, samples of a hop) of the kernels taken tap by tap; form -1: by another kernel."""
    v = [_c.c_int() for _ in range(4)]
    _check(lib().nna_plan_short_tiles(plan.handle, B, L, *(_c.byref(i) for i in v)))
    return tuple(i.value for i in v)


def nna_plan_mel_weights(plan: Plan) -> np.ndarray:
    i = plan.info()
    out = np.empty((i["out_bins"], i["bank_rows"] // 2), dtype=np.float64)
    _check(lib().nna_plan_mel_weights(plan.handle, out.ctypes.data_as(_c.POINTER(_c.c_double)), out.size))
    return out


def nna_plan_cqt_lengths(plan: Plan) -> np.ndarray:
    i = plan.info()
    # (out_bins counts (Re, Im) row pairs twice for a complex-output CQT plan; the plan's bank has 2 rows per bin)
    out = np.empty(i["out_bins"] if i["kind"] == NNA_KIND_CQT1992 else i["bank_rows"] // 2, dtype=np.int64)
    _check(lib().nna_plan_cqt_lengths(plan.handle, out.ctypes.data_as(_c.POINTER(_LL)), out.size))
    return out


def nna_plan_sigma(plan: Plan) -> np.ndarray:
    i = plan.info()
    out = np.empty(i["bank_rows"] // 2, dtype=np.float64)
    _check(lib().nna_plan_sigma(plan.handle, out.ctypes.data_as(_c.POINTER(_c.c_double)), out.size))
    return out


def _run(fn, plan: Plan, x, out, stream):
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()):
        raise TypeError("x must be a contiguous float32 CUDA tensor [B, L]")
    if x.dim() != 2:
        raise TypeError("x must be [B, L]")
    if x.device.index != plan.device:
        raise ValueError("x lives on a different device than the plan")
    B, L = x.shape
    bins, frames = nna_out_shape(plan, B, L)
    if out is None:
        out = torch.empty((B, bins, frames), dtype=torch.float32, device=x.device)
    elif not (out.is_cuda and out.dtype == torch.float32 and out.is_contiguous()
              and tuple(out.shape) == (B, bins, frames) and out.device == x.device):
        raise TypeError(f"out must be a contiguous float32 CUDA tensor of shape {(B, bins, frames)}")
    if stream is None:
        stream = torch.cuda.current_stream(x.device).cuda_stream
    _check(fn(plan.handle, x.data_ptr(), B, L, out.data_ptr(), stream))
    return out


def _run_octaves(cfn, plan: Plan, x, out, workspace, stream):
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dim() == 2):
        raise TypeError("x must be a contiguous float32 CUDA tensor [B, L]")
    need = nna_cqt2010v2_workspace(plan, x.shape[0], x.shape[1])
    if workspace is None:
        workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=x.device)
    elif not (workspace.is_cuda and workspace.is_contiguous() and workspace.device == x.device):
        raise TypeError("workspace must be a contiguous CUDA tensor on x's device")
    ws_bytes = workspace.numel() * workspace.element_size()

    def fn(handle, xp, B, L, op, st):
        return cfn(handle, xp, B, L, op, workspace.data_ptr(), ws_bytes, st)

    return _run(fn, plan, x, out, stream)


def nna_cqt2010v2(plan: Plan, x, out=None, workspace=None, stream=None):
    """out[B, n_bins, T] = constant-Q spectrogram of x[B, L] by recursive downsampling.  `workspace`: a CUDA
    tensor of at least nna_cqt2010v2_workspace(plan, B, L) bytes (one is made here if None)."""
    return _run_octaves(lib().nna_cqt2010v2, plan, x, out, workspace, stream)


NNA_STATIC_SCRATCH_BYTES = 64 << 20


def nna_cqt2010v2_static(plan: Plan, x, out=None, stream=None):
    """nna_cqt2010v2 with the library's own static workspace: the call allocates nothing (pass `out`)."""
    return _run(lib().nna_cqt2010v2_static, plan, x, out, stream)


def nna_cqt2010(plan: Plan, x, out=None, workspace=None, stream=None):
    """As nna_cqt2010v2, for a plan from nna_plan_cqt2010 (frequency-domain kernels per octave)."""
    return _run_octaves(lib().nna_cqt2010, plan, x, out, workspace, stream)


def nna_stft(plan: Plan, x, out=None, stream=None):
    """out[B, F, T] = STFT of x[B, L] (device tensors; asynchronous on `stream`); F = n_fft/2+1, or freq_bins
    for a plan from nna_plan_stft_scaled."""
    return _run(lib().nna_stft, plan, x, out, stream)


def nna_mel(plan: Plan, x, out=None, stream=None):
    """out[B, n_mels, T] = Mel spectrogram of x[B, L]."""
    return _run(lib().nna_mel, plan, x, out, stream)


def nna_mel_with_stft(plan: Plan, x, out=None, spec=None, stream=None):
    """(mel[B, n_mels, T], spec[B, n_fft/2+1, T]) from one contraction: the Mel spectrogram and the |X|^power
    spectrogram its filterbank is applied to."""
    import torch

    F = plan.constants()[1] // 2
    cfn = lib().nna_mel_with_stft
    holder = {}

    def fn(handle, xp, B, L, op, st):
        T = nna_out_shape(plan, B, L)[1]
        sp = spec
        if sp is None:
            sp = torch.empty((B, F, T), dtype=torch.float32, device=x.device)
        elif not (sp.is_cuda and sp.dtype == torch.float32 and sp.is_contiguous() and tuple(sp.shape) == (B, F, T)
                  and sp.device == x.device):
            raise TypeError(f"spec must be a contiguous float32 CUDA tensor of shape {(B, F, T)}")
        holder["spec"] = sp
        return cfn(handle, xp, B, L, op, sp.data_ptr(), st)

    mel = _run(fn, plan, x, out, stream)
    return mel, holder["spec"]


def nna_cqt_workspace(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_cqt_workspace(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_cqt_in_workspace(plan: Plan, x, workspace, out=None, stream=None):
    """nna_cqt or nna_cqt1992, by the plan's kind, in a CUDA tensor of the caller's."""
    if not (workspace.is_cuda and workspace.is_contiguous() and workspace.device == x.device):
        raise TypeError("workspace must be a contiguous CUDA tensor on x's device")
    ws_bytes = workspace.numel() * workspace.element_size()

    def fn(handle, xp, B, L, op, st):
        return lib().nna_cqt_in_workspace(handle, xp, B, L, op, workspace.data_ptr(), ws_bytes, st)

    return _run(fn, plan, x, out, stream)


def _memory_on(stream, need: int, device):
    """`need` bytes of the stream a call runs on (None: torch's current one), or None where they can't be that stream's alone: what its
    allocator hands out again when the call has returned is used behind the call."""
    import torch

    if stream is None and device.index == torch.cuda.current_device():
        return _outlives_capture(torch.empty(need, dtype=torch.uint8, device=device))
    # HIP's names for the default stream (1) and for every thread's own (2) are no streams that torch has an allocator for; a handle may also
    # come as a ctypes pointer
    if stream is not None and (not isinstance(stream, int) or stream in (1, 2)):
        return None
    # (ExternalStream takes 0, the default stream's handle, for "none given" and is then another stream, of torch's pool)
    on = (torch.cuda.current_stream(device) if stream is None else
          torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device))
    with torch.cuda.stream(on):
        return _outlives_capture(torch.empty(need, dtype=torch.uint8, device=device))


def _outlives_capture(memory):
    """`memory`, or None where the current stream is being captured and `memory` is not of a graph's own pool: a graph that torch knows
    nothing of would be replayed when its allocator has long handed the memory to others."""
    import torch

    if not torch.cuda.is_current_stream_capturing():
        return memory
    at = memory.data_ptr()
    pools = [s["segment_pool_id"] for s in torch.cuda.memory_snapshot() if s["address"] <= at < s["address"] + s["total_size"]]
    return memory if pools and tuple(pools[0]) != (0, 0) else None


def _run_one_rate(cfn, kind, plan, x, out, stream):
    """`cfn`, in a workspace where that is the faster way: memory of the stream the call runs on, back with its allocator
    when the call returns.  (Asking takes 0.8 us of host time, a call with memory 5 us more than one without: 8.4 and 12.8 us.)"""
    import torch

    def fn(handle, xp, B, L, op, st):
        need = nna_cqt_workspace(plan, B, L)
        if not need or plan.constants()[0] != kind:  # (nna_cqt_in_workspace takes either kind; `cfn` refuses the other's)
            return cfn(handle, xp, B, L, op, st)
        try:
            workspace = _memory_on(stream, need, x.device)
        except torch.OutOfMemoryError:
            workspace = None
        if workspace is None:
            return cfn(handle, xp, B, L, op, st)
        return lib().nna_cqt_in_workspace(handle, xp, B, L, op, workspace.data_ptr(), need, st)

    return _run(fn, plan, x, out, stream)


def nna_cqt1992(plan: Plan, x, out=None, stream=None):
    """out[B, n_bins, T] = constant-Q spectrogram of x[B, L] with frequency-domain kernels."""
    return _run_one_rate(lib().nna_cqt1992, NNA_KIND_CQT1992, plan, x, out, stream)


def nna_cqt(plan: Plan, x, out=None, stream=None):
    """out[B, n_bins, T] = constant-Q spectrogram of x[B, L]."""
    return _run_one_rate(lib().nna_cqt, NNA_KIND_CQT, plan, x, out, stream)


# ---- trainable Fourier kernels -------------------------------------------------------------------
def nna_plan_trainable(plan: Plan) -> Plan:
    _check(lib().nna_plan_trainable(plan.handle))
    return plan


def _bank_shape(plan: Plan):
    return plan.constants()[1:]


def _stream_of(t, stream):
    import torch

    return torch.cuda.current_stream(t.device).cuda_stream if stream is None else stream


def nna_plan_get_bank(plan: Plan, out=None, stream=None):
    """W[2F, K]: the plan's kernel bank as a float32 CUDA tensor (logical layout)."""
    import torch

    shape = _bank_shape(plan)
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=f"cuda:{plan.device}")
    elif not (out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == shape):
        raise TypeError(f"out must be a contiguous float32 CUDA tensor of shape {shape}")
    _check(lib().nna_plan_get_bank(plan.handle, out.data_ptr(), _stream_of(out, stream)))
    return out


def nna_plan_set_bank(plan: Plan, W, stream=None):
    shape = _bank_shape(plan)
    if not (W.is_cuda and W.dtype.is_floating_point and W.element_size() == 4 and W.is_contiguous()
            and tuple(W.shape) == shape and W.device.index == plan.device):
        raise TypeError(f"W must be a contiguous float32 CUDA tensor of shape {shape} on the plan's device")
    plan.bank_sets += 1
    _check(lib().nna_plan_set_bank(plan.handle, W.data_ptr(), _stream_of(W, stream)))


def nna_stft_backward_workspace(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_stft_backward_workspace(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_stft_backward(plan: Plan, x, gout, want_gw=True, want_gx=True, workspace=None, stream=None):
    """(gW[2F, K] or None, gx[B, L] or None) = gradients of a loss through nna_stft(plan, x), given
    gout[B, F, T] = dLoss/dout.  `workspace`: a CUDA tensor of nna_stft_backward_workspace bytes (made here if None)."""
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 2):
        raise TypeError("x must be a contiguous float32 CUDA tensor [B, L]")
    B, L = x.shape
    bins, frames = nna_out_shape(plan, B, L)
    if not (gout.is_cuda and gout.dtype == torch.float32 and gout.is_contiguous()
            and tuple(gout.shape) == (B, bins, frames) and gout.device == x.device):
        raise TypeError(f"gout must be a contiguous float32 CUDA tensor of shape {(B, bins, frames)}")
    need = nna_stft_backward_workspace(plan, B, L)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() * workspace.element_size()
    gw = torch.empty(_bank_shape(plan), dtype=torch.float32, device=x.device) if want_gw else None
    gx = torch.empty_like(x) if want_gx else None
    _check(lib().nna_stft_backward(plan.handle, x.data_ptr(), B, L, gout.data_ptr(),
                                   gw.data_ptr() if want_gw else None, gx.data_ptr() if want_gx else None,
                                   workspace.data_ptr(), ws_bytes, _stream_of(x, stream)))
    return gw, gx


def nna_cqt_backward_workspace(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_cqt_backward_workspace(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_cqt_backward(plan: Plan, x, gout, want_gw=True, want_gx=True, workspace=None, stream=None):
    """(gW[2 n_bins, n_taps] or None, gx[B, L] or None) = gradients of a loss through nna_cqt(plan, x), given
    gout = dLoss/dout.  `workspace`: a CUDA tensor of nna_cqt_backward_workspace bytes (made here if None)."""
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 2):
        raise TypeError("x must be a contiguous float32 CUDA tensor [B, L]")
    B, L = x.shape
    bins, frames = nna_out_shape(plan, B, L)
    if not (gout.is_cuda and gout.dtype == torch.float32 and gout.is_contiguous()
            and tuple(gout.shape) == (B, bins, frames) and gout.device == x.device):
        raise TypeError(f"gout must be a contiguous float32 CUDA tensor of shape {(B, bins, frames)}")
    need = nna_cqt_backward_workspace(plan, B, L)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() * workspace.element_size()
    gw = torch.empty(_bank_shape(plan), dtype=torch.float32, device=x.device) if want_gw else None
    gx = torch.empty_like(x) if want_gx else None
    _check(lib().nna_cqt_backward(plan.handle, x.data_ptr(), B, L, gout.data_ptr(),
                                  gw.data_ptr() if want_gw else None, gx.data_ptr() if want_gx else None,
                                  workspace.data_ptr(), ws_bytes, _stream_of(x, stream)))
    return gw, gx


def nna_cqt2010v2_backward_workspace(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_cqt2010v2_backward_workspace(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_cqt2010v2_backward(plan: Plan, x, gout, want_gw=True, want_gx=True, workspace=None, stream=None):
    """(gW[2 n_top, n_taps] or None, gx[B, L] or None) = gradients of a loss through nna_cqt2010v2(plan, x), given
    gout = dLoss/dout.  `workspace`: a CUDA tensor of nna_cqt2010v2_backward_workspace bytes (made here if None)."""
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 2):
        raise TypeError("x must be a contiguous float32 CUDA tensor [B, L]")
    B, L = x.shape
    bins, frames = nna_out_shape(plan, B, L)
    if not (gout.is_cuda and gout.dtype == torch.float32 and gout.is_contiguous()
            and tuple(gout.shape) == (B, bins, frames) and gout.device == x.device):
        raise TypeError(f"gout must be a contiguous float32 CUDA tensor of shape {(B, bins, frames)}")
    need = nna_cqt2010v2_backward_workspace(plan, B, L)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() * workspace.element_size()
    gw = torch.empty(_bank_shape(plan), dtype=torch.float32, device=x.device) if want_gw else None
    gx = torch.empty_like(x) if want_gx else None
    _check(lib().nna_cqt2010v2_backward(plan.handle, x.data_ptr(), B, L, gout.data_ptr(),
                                        gw.data_ptr() if want_gw else None, gx.data_ptr() if want_gx else None,
                                        workspace.data_ptr(), ws_bytes, _stream_of(x, stream)))
    return gw, gx


def _spectral_shapes(plan: Plan):
    """(shape of the spectral kernels Ysk, shape of the STFT stage's bank) of a plan with frequency-domain kernels"""
    i = (nna_plan_part(plan, 0) if plan.info()["kind"] == NNA_KIND_CQT2010 else plan).info()
    return (plan.spectral_rows, i["bank_rows"] // 2), (i["bank_rows"], i["taps"])


def nna_plan_get_spectral_kernels(plan: Plan, out=None, stream=None):
    """Ysk[2 n_bins, F]: the spectral kernels of a trainable plan from nna_plan_cqt1992 / nna_plan_cqt2010."""
    import torch

    shape = _spectral_shapes(plan)[0]
    if out is None:
        out = torch.empty(shape, dtype=torch.float32, device=f"cuda:{plan.device}")
    elif not (out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and tuple(out.shape) == shape):
        raise TypeError(f"out must be a contiguous float32 CUDA tensor of shape {shape}")
    _check(lib().nna_plan_get_spectral_kernels(plan.handle, out.data_ptr(), _stream_of(out, stream)))
    return out


def nna_plan_set_spectral_kernels(plan: Plan, Y, stream=None):
    shape = _spectral_shapes(plan)[0]
    if not (Y.is_cuda and Y.dtype.is_floating_point and Y.element_size() == 4 and Y.is_contiguous()
            and tuple(Y.shape) == shape and Y.device.index == plan.device):
        raise TypeError(f"Y must be a contiguous float32 CUDA tensor of shape {shape} on the plan's device")
    _check(lib().nna_plan_set_spectral_kernels(plan.handle, Y.data_ptr(), _stream_of(Y, stream)))


def _spectral_backward(name, plan, x, gout, want_gy, want_gw, want_gx, workspace, stream):
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 2):
        raise TypeError("x must be a contiguous float32 CUDA tensor [B, L]")
    B, L = x.shape
    bins, frames = nna_out_shape(plan, B, L)
    if not (gout.is_cuda and gout.dtype == torch.float32 and gout.is_contiguous()
            and tuple(gout.shape) == (B, bins, frames) and gout.device == x.device):
        raise TypeError(f"gout must be a contiguous float32 CUDA tensor of shape {(B, bins, frames)}")
    n = _c.c_size_t()
    _check(getattr(lib(), name + "_backward_workspace")(plan.handle, B, L, _c.byref(n)))
    if workspace is None:
        workspace = torch.empty(n.value, dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() * workspace.element_size()
    y_shape, w_shape = _spectral_shapes(plan)
    gy = torch.empty(y_shape, dtype=torch.float32, device=x.device) if want_gy else None
    gw = torch.empty(w_shape, dtype=torch.float32, device=x.device) if want_gw else None
    gx = torch.empty_like(x) if want_gx else None
    _check(getattr(lib(), name + "_backward")(plan.handle, x.data_ptr(), B, L, gout.data_ptr(),
                                              gy.data_ptr() if want_gy else None, gw.data_ptr() if want_gw else None,
                                              gx.data_ptr() if want_gx else None, workspace.data_ptr(), ws_bytes,
                                              _stream_of(x, stream)))
    return gy, gw, gx


def nna_cqt1992_backward_workspace(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_cqt1992_backward_workspace(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_cqt2010_backward_workspace(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_cqt2010_backward_workspace(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_cqt1992_backward(plan: Plan, x, gout, want_gy=True, want_gw=True, want_gx=True, workspace=None, stream=None):
    """(gYsk[2 n_bins, F], gW[2F, n_fft], gx[B, L]; None where not wanted) = gradients of a loss through
    nna_cqt1992(plan, x), given gout = dLoss/dout."""
    return _spectral_backward("nna_cqt1992", plan, x, gout, want_gy, want_gw, want_gx, workspace, stream)


def nna_cqt2010_backward(plan: Plan, x, gout, want_gy=True, want_gw=True, want_gx=True, workspace=None, stream=None):
    """As nna_cqt1992_backward, through nna_cqt2010(plan, x): the top octave's kernels are the weights of every octave."""
    return _spectral_backward("nna_cqt2010", plan, x, gout, want_gy, want_gw, want_gx, workspace, stream)


def _mel_shape(plan: Plan):
    i = plan.info()
    return (i["out_bins"], i["bank_rows"] // 2)


def nna_plan_get_mel_weights(plan: Plan, stream=None):
    """Wmel[n_mels, F]: the filterbank of a trainable Mel plan as a float32 CUDA tensor."""
    import torch

    out = torch.empty(_mel_shape(plan), dtype=torch.float32, device=f"cuda:{plan.device}")
    _check(lib().nna_plan_get_mel_weights(plan.handle, out.data_ptr(), _stream_of(out, stream)))
    return out


def nna_plan_set_mel_weights(plan: Plan, W, stream=None):
    shape = _mel_shape(plan)
    if not (W.is_cuda and W.element_size() == 4 and W.dtype.is_floating_point and W.is_contiguous()
            and tuple(W.shape) == shape and W.device.index == plan.device):
        raise TypeError(f"W must be a contiguous float32 CUDA tensor of shape {shape} on the plan's device")
    _check(lib().nna_plan_set_mel_weights(plan.handle, W.data_ptr(), _stream_of(W, stream)))


def nna_mel_backward_workspace(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_mel_backward_workspace(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_mel_backward(plan: Plan, x, gout, want_gmelw=True, want_gw=True, want_gx=True, workspace=None, stream=None):
    """(gWmel[n_mels, F], gW[2F, K], gx[B, L]) (None where not wanted) = gradients of a loss through
    nna_mel(plan, x), given gout[B, n_mels, T] = dLoss/dout."""
    import torch

    if not (isinstance(x, torch.Tensor) and x.is_cuda and x.dtype == torch.float32 and x.is_contiguous() and x.dim() == 2):
        raise TypeError("x must be a contiguous float32 CUDA tensor [B, L]")
    B, L = x.shape
    bins, frames = nna_out_shape(plan, B, L)
    if not (gout.is_cuda and gout.dtype == torch.float32 and gout.is_contiguous()
            and tuple(gout.shape) == (B, bins, frames) and gout.device == x.device):
        raise TypeError(f"gout must be a contiguous float32 CUDA tensor of shape {(B, bins, frames)}")
    need = nna_mel_backward_workspace(plan, B, L)
    if workspace is None:
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    ws_bytes = workspace.numel() * workspace.element_size()
    gm = torch.empty(_mel_shape(plan), dtype=torch.float32, device=x.device) if want_gmelw else None
    gw = torch.empty(_bank_shape(plan), dtype=torch.float32, device=x.device) if want_gw else None
    gx = torch.empty_like(x) if want_gx else None
    _check(lib().nna_mel_backward(plan.handle, x.data_ptr(), B, L, gout.data_ptr(),
                                  gm.data_ptr() if want_gmelw else None, gw.data_ptr() if want_gw else None,
                                  gx.data_ptr() if want_gx else None, workspace.data_ptr(), ws_bytes,
                                  _stream_of(x, stream)))
    return gm, gw, gx


def nna_kept_bytes(plan: Plan, B: int, L: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_kept_bytes(plan.handle, B, L, _c.byref(n)))
    return n.value


def nna_forward_keep(plan: Plan, x, stream=None, size=None, kept=None):
    """(out, kept): nna_stft, nna_mel or nna_cqt of a trainable plan, and what nna_backward_kept takes instead of computing it again.
    `size`: nna_kept_bytes of the call, where the caller has asked for it.  `kept`: a CUDA tensor of that many bytes to write it to (places that
    stand for no frame or no kernel are left as they are)."""
    import torch

    if size is None:
        size = nna_kept_bytes(plan, *x.shape)
    spec, given = None, kept
    if kept is None:
        kept = torch.empty(size, dtype=torch.uint8, device=x.device)
    elif not (kept.is_cuda and kept.is_contiguous() and kept.device == x.device and kept.numel() * kept.element_size() >= size):
        raise TypeError(f"kept must be a contiguous CUDA tensor of {size} bytes on x's device")
    kind, rows, _ = plan.constants()
    if kind == NNA_KIND_MEL:
        spec = torch.empty((x.shape[0], rows // 2, nna_out_shape(plan, *x.shape)[1]), dtype=torch.float32, device=x.device)

    def fn(handle, xp, B, L, op, st):
        return lib().nna_forward_keep(handle, xp, B, L, op, None if spec is None else spec.data_ptr(), kept.data_ptr(), size, st)

    out = _run(fn, plan, x, None, stream)
    if given is not None:
        _written(given)
    return out, kept


def nna_backward_kept(plan: Plan, x, gout, kept, want_gmelw=False, want_gw=True, want_gx=True, stream=None):
    """(gWmel or None, gW or None, gx or None), as the plan's backward call, with C from nna_forward_keep(plan, x)."""
    import torch

    for name, t in (("x", x), ("gout", gout)):
        if not (isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == torch.float32 and t.is_contiguous()):
            raise TypeError(f"{name} must be a contiguous float32 CUDA tensor")
    if x.dim() != 2 or not (kept.is_cuda and kept.is_contiguous() and gout.device == x.device == kept.device):
        raise TypeError("x must be [B, L], gout and kept contiguous on its device")
    B, L = x.shape
    bins, frames = nna_out_shape(plan, B, L)
    if tuple(gout.shape) != (B, bins, frames):
        raise TypeError(f"gout must be of shape {(B, bins, frames)}")
    kind = plan.constants()[0]
    size = nna_mel_backward_workspace if kind == NNA_KIND_MEL else nna_cqt_backward_workspace if kind == NNA_KIND_CQT else nna_stft_backward_workspace
    need = size(plan, B, L)
    workspace = torch.empty(need, dtype=torch.uint8, device=x.device)
    gm = torch.empty(_mel_shape(plan), dtype=torch.float32, device=x.device) if want_gmelw else None
    gw = torch.empty(_bank_shape(plan), dtype=torch.float32, device=x.device) if want_gw else None
    gx = torch.empty_like(x) if want_gx else None
    _check(lib().nna_backward_kept(plan.handle, x.data_ptr(), B, L, gout.data_ptr(), kept.data_ptr(), kept.numel() * kept.element_size(),
                                   gm.data_ptr() if want_gmelw else None, gw.data_ptr() if want_gw else None,
                                   gx.data_ptr() if want_gx else None, workspace.data_ptr(), need, _stream_of(x, stream)))
    return gm, gw, gx


# ---- operators of networks on the transforms' frames ------------------------------------------------------------------
NNA_F32, NNA_BF16, NNA_F16 = 0, 1, 2
NNA_BLOCK8 = 128
NNA_FRAMES_WIDTH = 2112  # bins of the frames that nna_layer_norm reads as the transforms write them
_types = {}
_current_stream = None
_increment_version = None


def _stream_on(device, stream):
    """The handle of torch's current stream on `device`, or `stream`.  (These operators' calls take ten microseconds where there is little to do: asking
    torch for the handle alone takes 0.1 us, for its stream object 2.1.)"""
    global _current_stream
    if stream is not None:
        return stream
    if _current_stream is None:
        import torch

        _current_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (lambda index: torch.cuda.current_stream(index).cuda_stream)
    return _current_stream(device.index)


def _under(stream, device, call):
    """call() with `stream` as torch's current one, or None where it is that already or none that torch has an allocator for: what the call allocates is then memory of
    the stream it is written on, and what it returns is not handed out again before the stream that it is returned to has done with it, too."""
    import torch

    if not isinstance(stream, int) or stream in (1, 2):  # (HIP's names for the default stream and for every thread's own; a ctypes pointer)
        return None
    current = torch.cuda.current_stream(device)
    if stream == current.cuda_stream:
        return None
    with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)):
        result = call()
    for t in result if isinstance(result, tuple) else (result,):
        for t in (t.stats, t.codes, t.scales) if isinstance(t, NormKept) else (t,):
            if t is not None:
                t.record_stream(current)
    return result


def _type_of(t, name, allowed=("float32", "bfloat16", "float16")):
    """The nna_dtype of a CUDA tensor, which is refused if it is none or of a type not `allowed`."""
    import torch

    if not _types:
        _types.update({torch.float32: (NNA_F32, "float32"), torch.bfloat16: (NNA_BF16, "bfloat16"), torch.float16: (NNA_F16, "float16")})
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise TypeError(f"{name} must be a CUDA tensor")
    known = _types.get(t.dtype)
    if known is None or known[1] not in allowed:
        raise TypeError(f"{name} must be of {' or '.join(allowed)}, not {t.dtype}")
    return known[0]


def _vector(t, name, shape, device, none=False):
    """The pointer of a contiguous float32 tensor of `shape` on `device` (None where that is allowed)."""
    import torch

    if t is None and none:
        return None
    if not (isinstance(t, torch.Tensor) and t.dtype == torch.float32 and t.is_contiguous() and t.shape == shape and t.device == device):
        raise TypeError(f"{name} must be a contiguous float32 tensor of shape {tuple(shape)} on {device}")
    return t.data_ptr()


def _written(*tensors):
    """Tells autograd of tensors of the caller's that a call has written through their pointers, as torch's own in-place operations do: a graph that
    holds one of them for its backward pass then refuses to run on the new values.  (0.3 us a tensor.)"""
    global _increment_version
    if _increment_version is None:
        from torch.autograd.graph import increment_version as _increment_version
    for t in tensors:
        if t is not None:
            _increment_version(t)


def _all_written(tensors):
    """_written of a list, in one call."""
    _written()
    _increment_version(tensors)


def _bytes_of(t):
    """The addresses from a tensor's first element to its last."""
    if not t.numel():
        return 0, 0
    at = t.data_ptr()
    return at, at + (sum((n - 1) * s for n, s in zip(t.shape, t.stride())) + 1) * t.element_size()


def _overlap(a, b):
    (a0, a1), (b0, b1) = _bytes_of(a), _bytes_of(b)
    return a0 < b1 and b0 < a1


def _refuse_overlap(out, *inputs):
    """A given output is written while other workgroups still read the inputs."""
    for t in inputs:
        if t is not None and _overlap(out, t):
            raise ValueError("out must not share memory with an input")


def _row_stride(x):
    """Elements between the rows of x[..., width] if its rows are at one distance from each other, or None."""
    shape, strides = x.shape, x.stride()
    if not x.numel():
        return shape[-1]
    if shape[-1] != 1 and strides[-1] != 1:
        return None
    step = far = None
    for n, s in zip(reversed(shape[:-1]), reversed(strides[:-1])):
        if n == 1:
            continue
        if step is None:
            step, far = s, s * n
        elif s != far:
            return None
        else:
            far = s * n
    return shape[-1] if step is None else step


def _workspace_on(stream, need, workspace, device):
    import torch

    if workspace is None:
        workspace = _memory_on(stream, need, device)
        if workspace is None:
            raise ValueError("torch has no allocator for this stream, or knows nothing of its capture: pass `workspace`")
    elif not (isinstance(workspace, torch.Tensor) and workspace.is_cuda and workspace.is_contiguous() and workspace.device == device):
        raise TypeError("workspace must be a contiguous CUDA tensor on the inputs' device")
    return workspace


class NormKept:
    """What nna_layer_norm keeps for nna_layer_norm_backward: every row's mean and 1 / sqrt(variance + eps) (`stats`), and the input
    itself (`x`) or its 8 bits (`codes`, `scales`)."""

    __slots__ = ("shape", "dtype", "out_dtype", "rows", "row_stride", "x", "stats", "codes", "scales")

    def tensors(self):
        return tuple(t for t in (self.x, self.stats, self.codes, self.scales) if t is not None)

    def with_tensors(self, tensors, bits):
        """The same with what tensors() gave (kept 8 or 32 `bits`)."""
        kept = NormKept()
        kept.shape, kept.dtype, kept.out_dtype, kept.rows, kept.row_stride = self.shape, self.dtype, self.out_dtype, self.rows, self.row_stride
        kept.x, kept.stats, kept.codes, kept.scales = (*tensors, None, None) if bits == 32 else (None, *tensors)
        return kept


def nna_layer_norm(x, weight=None, bias=None, eps=1e-5, out_dtype=None, keep=0, out=None, stream=None):
    """Layer norm over the last axis of x[..., width]: (x - mean) / sqrt(variance + eps) * weight + bias, contiguous, of x's type (float32 input:
    also of `out_dtype` bfloat16 or float16).  x's rows lie at one distance from each other, or x is frames as the transforms write
    them, ``spec.transpose(1, 2)`` of a contiguous float32 spec[B, bins, T].  weight, bias: float32 [width].
    keep: 0, or what is kept for nna_layer_norm_backward, returned behind y as a NormKept: 32 the input as it is, 8 the input in 8 bits
    (nna_pack8's; rows only, y of x's type).  `out` may be x itself, of contiguous rows and x's type, unless x is what is kept."""
    import torch

    xt = _type_of(x, "x")
    if stream is not None and (done := _under(stream, x.device, lambda: nna_layer_norm(x, weight, bias, eps, out_dtype, keep, out))) is not None:
        return done
    if x.dim() < 1:
        raise TypeError("x must have an axis to normalise")
    if keep not in (0, 8, 32):
        raise ValueError("keep: 0, 8 or 32")
    shape, width, device = x.shape, x.shape[-1], x.device
    out_dtype, given = x.dtype if out_dtype is None else out_dtype, out
    if out is None:
        out = torch.empty_like(x, dtype=out_dtype, memory_format=torch.contiguous_format)
    elif not (isinstance(out, torch.Tensor) and out.device == device and out.dtype == out_dtype and out.is_contiguous() and out.shape == shape):
        raise TypeError(f"out must be a contiguous {out_dtype} CUDA tensor of shape {tuple(shape)}")
    if given is not None and keep == 32 and _overlap(out, x):
        raise ValueError("keep=32 keeps x itself: out must not share its memory")
    yt = _type_of(out, "out")
    w, b = _vector(weight, "weight", (width,), device, none=True), _vector(bias, "bias", (width,), device, none=True)
    if given is not None:  # (over x only where every row is written where it was read, by the lanes that read it)
        _refuse_overlap(out, weight, bias, None if x.is_contiguous() and x.dtype == out_dtype and x.data_ptr() == out.data_ptr() else x)
    rows = x.numel() // width if width else 0
    step = _row_stride(x)
    kept = stats = codes = scales = None
    if keep:
        stats = x.new_empty((rows, 2), dtype=torch.float32)
        if keep == 8:
            codes = torch.empty((rows, width), dtype=torch.int8, device=device)
            scales = torch.empty((rows, -(-width // NNA_BLOCK8)), dtype=torch.float32, device=device)
        kept = NormKept()
        kept.shape, kept.dtype, kept.out_dtype, kept.rows, kept.row_stride = shape, x.dtype, out_dtype, rows, step
        kept.x, kept.stats, kept.codes, kept.scales = x if keep == 32 else None, stats, codes, scales
    sp, st = stats.data_ptr() if keep else None, _stream_on(x.device, stream)
    if step is not None:
        _check(lib().nna_layer_norm(x.data_ptr(), xt, rows, width, step, w, b, eps, out.data_ptr(), yt, sp,
                                    codes.data_ptr() if keep == 8 else None, scales.data_ptr() if keep == 8 else None, device.index, st))
    elif x.dim() == 3 and xt == NNA_F32 and (x.stride() == (width * shape[1], 1, shape[1]) or x.transpose(1, 2).is_contiguous()):
        if keep == 8:
            raise TypeError("keep=8: x must be rows (consecutive values next to each other)")
        _check(lib().nna_layer_norm_frames(x.data_ptr(), shape[0], width, shape[1], w, b, eps, out.data_ptr(), yt, sp, device.index, st))
    else:
        raise TypeError("x must be rows at one distance from each other, or the transpose of a contiguous float32 [B, bins, T]")
    if given is not None:
        _written(given)
    return (out, kept) if keep else out


def nna_layer_norm_backward(gout, kept, weight=None, want_gx=True, want_gw=True, workspace=None, stream=None):
    """(gx, gweight, gbias), None where not wanted: the gradients of a loss through nna_layer_norm(x, weight, bias, keep=...), given gout =
    dLoss/dy of y's shape and type and what that call kept.  gx is of x's type, laid out as x was read (rows contiguous).
    `workspace`: a CUDA tensor of nna_layer_norm_backward_workspace bytes (taken here if None)."""
    import torch

    gt = _type_of(gout, "gout")
    if stream is not None and (done := _under(stream, gout.device, lambda: nna_layer_norm_backward(gout, kept, weight, want_gx, want_gw, workspace))) is not None:
        return done
    if gout.dtype != kept.out_dtype or gout.shape != kept.shape or not gout.is_contiguous() or gout.device != kept.stats.device:
        raise TypeError(f"gout must be a contiguous {kept.out_dtype} CUDA tensor of shape {tuple(kept.shape)}")
    shape, width, device, rows = kept.shape, kept.shape[-1], gout.device, kept.rows
    w = _vector(weight, "weight", (width,), device, none=True)
    frames = kept.row_stride is None
    B, T = (shape[0], shape[1]) if frames else (0, 0)
    gx = gw = gb = None
    if want_gx:
        gx = kept.x.new_empty_strided(shape, (width * T, 1, T)) if frames else torch.empty_like(gout, dtype=kept.dtype)
    need = 0
    if want_gw:
        gw, gb = kept.stats.new_empty(width), kept.stats.new_empty(width)
        need = nna_layer_norm_backward_workspace(rows, width, B, T)
        workspace = _workspace_on(stream, need, workspace, device)
    ws = (workspace.data_ptr(), workspace.numel() * workspace.element_size()) if want_gw else (None, 0)
    grads = (gx.data_ptr() if want_gx else None, gw.data_ptr() if want_gw else None, gb.data_ptr() if want_gw else None)
    sp, st = kept.stats.data_ptr(), _stream_on(device, stream)
    if frames:
        _check(lib().nna_layer_norm_frames_backward(gout.data_ptr(), gt, kept.x.data_ptr(), B, width, T, sp, w, *grads, *ws, device.index, st))
    else:
        xt = {torch.float32: NNA_F32, torch.bfloat16: NNA_BF16, torch.float16: NNA_F16}[kept.dtype]
        codes, scales = kept.codes, kept.scales
        _check(lib().nna_layer_norm_backward(gout.data_ptr(), gt, None if kept.x is None else kept.x.data_ptr(), xt, rows, width, kept.row_stride,
                                             None if codes is None else codes.data_ptr(), None if scales is None else scales.data_ptr(), sp, w,
                                             *grads, *ws, device.index, st))
    return gx, gw, gb


def nna_layer_norm_backward_workspace(rows: int, width: int, B: int = 0, T: int = 0) -> int:
    """Bytes for `rows` rows, or for the frames of [B, width, T] (rows = B T)."""
    n = _c.c_size_t()
    _check(lib().nna_layer_norm_backward_workspace(rows, width, B, T, _c.byref(n)))
    return n.value


def nna_pack8(x, stream=None):
    """(codes int8 [..., width], scales float32 [..., ceil(width / 128)]): x[..., width] in 8 bits, 128 neighbours to a scale."""
    import torch

    xt = _type_of(x, "x")
    if stream is not None and (done := _under(stream, x.device, lambda: nna_pack8(x))) is not None:
        return done
    step = _row_stride(x) if x.dim() else None
    if step is None:
        raise TypeError("x must be rows at one distance from each other")
    width = x.shape[-1]
    codes = torch.empty_like(x, dtype=torch.int8, memory_format=torch.contiguous_format)
    scales = x.new_empty((*x.shape[:-1], -(-width // NNA_BLOCK8)), dtype=torch.float32)
    _check(lib().nna_pack8(x.data_ptr(), xt, x.numel() // width if width else 0, width, step, codes.data_ptr(), scales.data_ptr(), x.device.index,
                           _stream_on(x.device, stream)))
    return codes, scales


def nna_unpack8(codes, scales, dtype=None, out=None, stream=None):
    """The values that nna_pack8's codes stand for, codes * scales, in `dtype` (float32 if None), contiguous."""
    import torch

    if not (isinstance(codes, torch.Tensor) and codes.is_cuda and codes.dtype == torch.int8 and codes.is_contiguous() and codes.dim()):
        raise TypeError("codes must be a contiguous int8 CUDA tensor")
    if stream is not None and (done := _under(stream, codes.device, lambda: nna_unpack8(codes, scales, dtype, out))) is not None:
        return done
    width = codes.shape[-1]
    sp, given = _vector(scales, "scales", (*codes.shape[:-1], -(-width // NNA_BLOCK8)), codes.device), out
    if out is None:
        out = torch.empty_like(codes, dtype=torch.float32 if dtype is None else dtype)
    elif not (out.is_contiguous() and out.shape == codes.shape and out.device == codes.device and dtype in (None, out.dtype)):
        raise TypeError(f"out must be a contiguous CUDA tensor of shape {tuple(codes.shape)}")
    ot = _type_of(out, "out")
    if given is not None:
        _refuse_overlap(out, codes, scales)
    _check(lib().nna_unpack8(codes.data_ptr(), sp, codes.numel() // width if width else 0, width, out.data_ptr(), ot, codes.device.index,
                             _stream_on(codes.device, stream)))
    if given is not None:
        _written(given)
    return out


_strides3, _strides2 = _LL * 3, _LL * 2


def _heads(q, k, v, axes):
    """(nna_dtype, sizes, the arguments q, k, v stand for) of [B, (T,) H, d] tensors; their strides but for the last are their own."""
    import torch

    t, tensor, dtype, device = _type_of(q, "q", ("float32", "bfloat16")), torch.Tensor, q.dtype, q.device
    if not (isinstance(k, tensor) and isinstance(v, tensor) and k.dtype == dtype and v.dtype == dtype and k.device == device and v.device == device):
        raise TypeError("q, k and v must be tensors of one type, on one device")
    shape, wide = q.shape, v.shape
    if len(shape) != axes or k.shape != shape or len(wide) != axes or wide[:-1] != shape[:-1]:
        raise TypeError("q and k must be " + ("[B, T, H, dk] and v [B, T, H, dv]" if axes == 4 else "[B, H, dk] and v [B, H, dv]"))
    dk, dv, array = shape[-1], wide[-1], _strides3 if axes == 4 else _strides2
    (*sq, lq), (*sk, lk), (*sv, lv) = q.stride(), k.stride(), v.stride()
    if (dk != 1 and (lq != 1 or lk != 1)) or (dv != 1 and lv != 1):
        raise TypeError("a head's values must lie next to each other")
    return t, (*shape, dv), (q.data_ptr(), array(*sq), k.data_ptr(), array(*sk), v.data_ptr(), array(*sv))


def _lengths(lengths, B, device):
    import torch

    if lengths is None:
        return None
    if not (isinstance(lengths, torch.Tensor) and lengths.dtype == torch.int32 and lengths.is_contiguous() and tuple(lengths.shape) == (B,) and lengths.device == device):
        raise TypeError(f"lengths must be a contiguous int32 tensor of shape {(B,)} on {device}")
    return lengths.data_ptr()


def nna_decay_attention_workspace(B: int, T: int, H: int, dk: int, dv: int) -> int:
    """Bytes that nna_decay_attention needs; 0 where there are sequences and heads enough to fill the card."""
    n = _c.c_size_t()
    _check(lib().nna_decay_attention_workspace(B, T, H, dk, dv, _c.byref(n)))
    return n.value


def nna_decay_attention_backward_workspace(B: int, T: int, H: int, dk: int, dv: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_decay_attention_backward_workspace(B, T, H, dk, dv, _c.byref(n)))
    return n.value


def nna_decay_attention(q, k, v, decay, scale=None, state=None, lengths=None, want_state=False, out=None, workspace=None, stream=None):
    """o[B, T, H, dv] of linear attention with a decay for each head, S_t = decay S_{t-1} + k_t^T v_t, o_t = scale q_t S_t; with `want_state`
    (o, S after the last frame [B, H, dk, dv]).  q, k [B, T, H, dk], v [B, T, H, dv]: float32 or bfloat16, any strides but the last.  decay: float32 [H], in
    [0, 1].  scale: dk**-0.5 if None.  state: float32 [B, H, dk, dv] before the first frame (None: zero).  lengths: int32 [B] on the GPU; frames
    from there on take no part, and their outputs are zero.  `workspace`: nna_decay_attention_workspace bytes, 256-byte aligned (taken here if None)."""
    import torch

    t, (B, T, H, dk, dv), args = _heads(q, k, v, 4)
    device = q.device
    if stream is not None and (done := _under(stream, device, lambda: nna_decay_attention(q, k, v, decay, scale, state, lengths, want_state, out, workspace))) is not None:
        return done
    dp, sp, lp = _vector(decay, "decay", (H,), device), _vector(state, "state", (B, H, dk, dv), device, none=True), _lengths(lengths, B, device)
    given = out
    if out is None:
        out = q.new_empty((B, T, H, dv))
    elif not (isinstance(out, torch.Tensor) and out.dtype == q.dtype and out.is_contiguous() and tuple(out.shape) == (B, T, H, dv) and out.device == device):
        raise TypeError(f"out must be a contiguous {q.dtype} tensor of shape {(B, T, H, dv)}")
    else:
        _refuse_overlap(out, q, k, v, decay, state, lengths)
    last = decay.new_empty((B, H, dk, dv)) if want_state else None
    need = nna_decay_attention_workspace(B, T, H, dk, dv)
    ws = (None, 0)
    if need:
        workspace = _workspace_on(stream, need, workspace, device)
        ws = (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _check(lib().nna_decay_attention(*args, t, B, T, H, dk, dv, dp, dk**-0.5 if scale is None else scale, lp, sp, last.data_ptr() if want_state else None,
                                     out.data_ptr(), *ws, device.index, _stream_on(device, stream)))
    if given is not None:
        _written(given)
    return (out, last) if want_state else out


def nna_decay_attention_backward(gout, q, k, v, decay, scale=None, state=None, lengths=None, gstate=None, want_gstate=False, workspace=None, stream=None):
    """(gq, gk, gv, gradient of the first state or None): the gradients of a loss through nna_decay_attention, given gout = dLoss/do (contiguous)
    and gstate = dLoss/d(last state) (None: zero).  `workspace`: nna_decay_attention_backward_workspace bytes (taken here if None)."""
    import torch

    t, (B, T, H, dk, dv), args = _heads(q, k, v, 4)
    device = q.device
    if stream is not None and (done := _under(stream, device, lambda: nna_decay_attention_backward(gout, q, k, v, decay, scale, state, lengths, gstate, want_gstate,
                                                                                                   workspace))) is not None:
        return done
    dp, sp, lp = _vector(decay, "decay", (H,), device), _vector(state, "state", (B, H, dk, dv), device, none=True), _lengths(lengths, B, device)
    lastp = _vector(gstate, "gstate", (B, H, dk, dv), device, none=True)
    if not (isinstance(gout, torch.Tensor) and gout.dtype == q.dtype and gout.is_contiguous() and tuple(gout.shape) == (B, T, H, dv) and gout.device == device):
        raise TypeError(f"gout must be a contiguous {q.dtype} tensor of shape {(B, T, H, dv)}")
    gq, gk, gv = q.new_empty((B, T, H, dk)), q.new_empty((B, T, H, dk)), torch.empty_like(gout)
    first = decay.new_empty((B, H, dk, dv)) if want_gstate else None
    need = nna_decay_attention_backward_workspace(B, T, H, dk, dv)
    ws = (None, 0)
    if need:
        workspace = _workspace_on(stream, need, workspace, device)
        ws = (workspace.data_ptr(), workspace.numel() * workspace.element_size())
    _check(lib().nna_decay_attention_backward(gout.data_ptr(), *args, t, B, T, H, dk, dv, dp, dk**-0.5 if scale is None else scale, lp, sp, lastp,
                                              gq.data_ptr(), gk.data_ptr(), gv.data_ptr(), first.data_ptr() if want_gstate else None, *ws,
                                              device.index, _stream_on(device, stream)))
    return gq, gk, gv, first


def nna_decay_attention_step(q, k, v, decay, state, scale=None, out=None, stream=None):
    """o[B, H, dv] of one new frame q, k [B, H, dk], v [B, H, dv] of each sequence; state float32 [B, H, dk, dv] is updated in place."""
    import torch

    t, (B, H, dk, dv), args = _heads(q, k, v, 3)
    device = q.device
    if stream is not None and (done := _under(stream, device, lambda: nna_decay_attention_step(q, k, v, decay, state, scale, out))) is not None:
        return done
    dp, sp = _vector(decay, "decay", (H,), device), _vector(state, "state", (B, H, dk, dv), device)
    given = out
    if out is None:
        out = q.new_empty((B, H, dv))
    elif not (isinstance(out, torch.Tensor) and out.dtype == q.dtype and out.is_contiguous() and tuple(out.shape) == (B, H, dv) and out.device == device):
        raise TypeError(f"out must be a contiguous {q.dtype} tensor of shape {(B, H, dv)}")
    else:
        _refuse_overlap(out, q, k, v, decay, state)
    _check(lib().nna_decay_attention_step(*args, t, B, H, dk, dv, dp, dk**-0.5 if scale is None else scale, sp, out.data_ptr(), device.index,
                                          _stream_on(device, stream)))
    _written(state, given)
    return out


def nna_rotary_freqs(width, base=10000.0, scale=1.0, device=0):
    """float64 [width // 2] on the GPU: radians a position for nna_rotate_heads, base^(-2 i / width) / scale, of heads whose first `width` values (even) are rotated.
    `scale` above 1 stretches positions for contexts longer than those trained on; another `base` stretches the slow pairs alone.  Any other rule is its own tensor."""
    import torch

    width = int(width)
    if width < 0 or width % 2:
        raise ValueError("width must be even")
    if not (base > 0 and scale > 0 and np.isfinite(base) and np.isfinite(scale)):
        raise ValueError("base and scale must be positive")
    return torch.from_numpy(float(base) ** (-np.arange(0, width, 2, dtype=np.float64) / max(1, width)) / float(scale)).to(device if device is not None else "cpu")


def _turns(q, k, freqs, positions, offset, q_weight, k_weight, eps):
    """(nna_dtype, (B, T, width), [q, strides, heads, k, strides, heads], the arguments from freqs to the weights) of q, k [B, (T,) heads, width]."""
    import torch

    t, tensor, device, dtype, shape = _type_of(q, "q"), torch.Tensor, q.device, q.dtype, q.shape
    one = len(shape) == 3
    if one:
        (B, H, width), T, (sb, sh, last) = shape, 1, q.stride()
        args = [q.data_ptr(), _strides3(sb, 0, sh), H]
    elif len(shape) == 4:
        (B, T, H, width), (sb, st, sh, last) = shape, q.stride()
        args = [q.data_ptr(), _strides3(sb, st, sh), H]
    else:
        raise TypeError("q must be [B, T, heads, width], or [B, heads, width] of one frame")
    if k is None:
        args += (None, None, 0)
    else:
        if not (isinstance(k, tensor) and k.dtype == dtype and k.device == device and len(k.shape) == len(shape)):
            raise TypeError("k must be of q's type, on its device and of its shape but for the number of heads")
        heads = k.shape[-2]
        if k.shape != ((B, heads, width) if one else (B, T, heads, width)):
            raise TypeError("k must be of q's type, on its device and of its shape but for the number of heads")
        sb, *st, sh, last_k = k.stride()
        last = last if last != 1 else last_k
        args += (k.data_ptr(), _strides3(sb, 0 if one else st[0], sh), heads)
    if last != 1 and width != 1:
        raise TypeError("a head's values must lie next to each other")
    if not (isinstance(freqs, tensor) and freqs.dtype == torch.float64 and freqs.dim() == 1 and freqs.is_contiguous() and freqs.device == device):
        raise TypeError(f"freqs must be a contiguous float64 tensor of one axis on {device}")
    at, steps = None, None
    if positions is not None:
        if not (isinstance(positions, tensor) and positions.dtype == torch.int32 and positions.device == device and positions.shape == ((B,) if one else (B, T))):
            raise TypeError(f"positions must be an int32 tensor of shape {(B,) if one else (B, T)} on {device}")
        if offset:
            raise ValueError("offset is where positions are not given")
        at, steps = positions.data_ptr(), _strides2(positions.stride(0), 0) if one else _strides2(*positions.stride())
    norm = eps is not None
    if not norm and (q_weight is not None or k_weight is not None):
        raise ValueError("weights are the norm's: give eps")
    weights = (_vector(q_weight, "q_weight", (width,), device, none=True), _vector(k_weight, "k_weight", (width,), device, none=True))
    return t, (B, T, width), args, (freqs.data_ptr(), freqs.numel(), at, steps, int(offset), norm, eps if norm else 0.0, *weights)


def nna_rotate_heads(q, k, freqs, positions=None, offset=0, q_weight=None, k_weight=None, eps=None, interleaved=False, out=None, stream=None):
    """(q, k) with each head normalised by its root mean square (`eps` given; times q_weight, k_weight, float32 [width]) and the pairs of its first 2 len(freqs) values
    rotated by position * freqs, contiguous.  q [B, T, heads, width], k [B, T, its own heads, width] or None; or [B, heads, width] of one frame: float32, bfloat16 or float16,
    any strides but the last.  freqs: float64 (nna_rotary_freqs).  positions: int32 [B, T] ([B]) on the GPU; if None, frame t is at offset + t.  Pair j is (j, j + len(freqs)), or
    `interleaved` (2 j, 2 j + 1).  out: (q, k) to write to, not over inputs."""
    import torch

    t, (B, T, width), args, (freqs_p, pairs, *rest) = _turns(q, k, freqs, positions, offset, q_weight, k_weight, eps)
    device = q.device
    if stream is not None and (done := _under(stream, device, lambda: nna_rotate_heads(q, k, freqs, positions, offset, q_weight, k_weight, eps, interleaved, out))) is not None:
        return done
    if out is None:
        yq, yk = torch.empty_like(q, memory_format=torch.contiguous_format), None if k is None else torch.empty_like(k, memory_format=torch.contiguous_format)
    else:
        yq, yk = out
        for y, x in ((yq, q), (yk, k)):
            if (y is None) != (x is None) or (y is not None and not (y.dtype == x.dtype and y.is_contiguous() and y.shape == x.shape and y.device == device)):
                raise TypeError("out must be contiguous tensors of q's and k's shapes and type")
            if y is not None:
                _refuse_overlap(y, q, k, freqs, positions, q_weight, k_weight)
        if yk is not None and _overlap(yq, yk):
            raise ValueError("the outputs must not share memory")
    _check(lib().nna_rotate_heads(*args, t, B, T, width, freqs_p, pairs, bool(interleaved), *rest, yq.data_ptr(), None if yk is None else yk.data_ptr(), device.index,
                                  _stream_on(device, stream)))
    if out is not None:
        _written(yq, yk)
    return yq, yk


def nna_rotate_heads_backward_workspace(B: int, T: int, width: int) -> int:
    n = _c.c_size_t()
    _check(lib().nna_rotate_heads_backward_workspace(B, T, width, _c.byref(n)))
    return n.value


def nna_rotate_heads_backward(gq, gk, q, k, freqs, positions=None, offset=0, q_weight=None, k_weight=None, eps=None, interleaved=False, want_weights=True,
                              workspace=None, stream=None):
    """(gradient of q, of k, of q_weight, of k_weight; None where there is none or not wanted) of a loss through nna_rotate_heads, given gq, gk = dLoss/d(its outputs), contiguous.
    The weights' are those of ones where they are not given.  `workspace`: nna_rotate_heads_backward_workspace bytes (taken here if None)."""
    import torch

    t, (B, T, width), args, (freqs_p, pairs, *rest) = _turns(q, k, freqs, positions, offset, q_weight, k_weight, eps)
    device = q.device
    if stream is not None and (done := _under(stream, device, lambda: nna_rotate_heads_backward(gq, gk, q, k, freqs, positions, offset, q_weight, k_weight, eps, interleaved,
                                                                                                want_weights, workspace))) is not None:
        return done
    for g, x in ((gq, q), (gk, k)):
        if (g is None) != (x is None) or (g is not None and not (isinstance(g, torch.Tensor) and g.dtype == x.dtype and g.is_contiguous() and g.shape == x.shape
                                                                 and g.device == device)):
            raise TypeError("gq and gk must be contiguous tensors of q's and k's shapes and type")
    hq, hk = torch.empty_like(gq), None if k is None else torch.empty_like(gk)
    gqw = gkw = None
    ws = (None, 0)
    if want_weights and eps is not None:
        gqw = torch.empty(width, dtype=torch.float32, device=device)
        gkw = None if k is None else torch.empty(width, dtype=torch.float32, device=device)
        need = nna_rotate_heads_backward_workspace(B, T, width)
        workspace = _workspace_on(stream, need, workspace, device)
        ws = (workspace.data_ptr(), workspace.numel() * workspace.element_size())

    def at(x):
        return None if x is None else x.data_ptr()

    _check(lib().nna_rotate_heads_backward(gq.data_ptr(), at(gk), *args, t, B, T, width, freqs_p, pairs, bool(interleaved), *rest, hq.data_ptr(), at(hk), at(gqw), at(gkw),
                                           *ws, device.index, _stream_on(device, stream)))
    return hq, hk, gqw, gkw


NNA_SCAN_KEPT = 64


def _gates(x, forget, input, axes):
    """(nna_dtype, x's shape, [x, strides, forget, strides, input, strides]) of [B, (T,) C] tensors."""
    import torch

    t, dtype, device, shape = _type_of(x, "x"), x.dtype, x.device, x.shape
    if len(shape) != axes:
        raise TypeError("x must be " + ("[B, T, C]" if axes == 3 else "[B, C]"))
    args = []
    for n, g in enumerate((x, forget, input)):
        if g is None and n == 2:
            args += (None, None if axes == 3 else 0)
            continue
        if g is not x and not (isinstance(g, torch.Tensor) and g.dtype == dtype and g.device == device and g.shape == shape):
            raise TypeError("forget and input must be of x's type and shape, on its device")
        *s, last = g.stride()
        if last != 1 and shape[-1] != 1:
            raise TypeError("a frame's channels must lie next to each other")
        args += (g.data_ptr(), _strides2(*s) if axes == 3 else s[0])
    return t, shape, args


def nna_gated_scan_workspace(B: int, T: int, C: int) -> int:
    """Bytes that nna_gated_scan and nna_gated_scan_backward need; 0 where there are sequences and channels enough to fill the card."""
    n = _c.c_size_t()
    _check(lib().nna_gated_scan_workspace(B, T, C, _c.byref(n)))
    return n.value


def _scan_workspace(B, T, C, workspace, device, stream):
    need = nna_gated_scan_workspace(B, T, C)
    if not need:
        return None, (None, 0)
    workspace = _workspace_on(stream, need, workspace, device)
    return workspace, (workspace.data_ptr(), workspace.numel() * workspace.element_size())


def nna_gated_scan(x, forget, input=None, state=None, lengths=None, want_state=False, keep=False, out=None, workspace=None, stream=None):
    """h[B, T, C] of the gated recurrence h_t = a_t h_{t-1} + u_t x_t, a = sigmoid(forget), u = sigmoid(input), or 1 - a where input is None; with `want_state` also the state after
    the last frame, float32 [B, C], with `keep` also what nna_gated_scan_backward takes (the states before every 64th frame).  x, forget, input [B, T, C]: float32, bfloat16 or
    float16, any strides but the last.  state: float32 [B, C] before the first frame (None: zero).  lengths: int32 [B] on the GPU; frames from there on take no part, and their
    outputs are zero.  `workspace`: nna_gated_scan_workspace bytes, 256-byte aligned (taken here if None)."""
    import torch

    t, (B, T, C), args = _gates(x, forget, input, 3)
    device = x.device
    if stream is not None and (done := _under(stream, device, lambda: nna_gated_scan(x, forget, input, state, lengths, want_state, keep, out, workspace))) is not None:
        return done
    sp, lp = _vector(state, "state", (B, C), device, none=True), _lengths(lengths, B, device)
    given = out
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    elif not (isinstance(out, torch.Tensor) and out.dtype == x.dtype and out.is_contiguous() and out.shape == x.shape and out.device == device):
        raise TypeError(f"out must be a contiguous {x.dtype} tensor of shape {(B, T, C)}")
    else:
        _refuse_overlap(out, x, forget, input, state, lengths)
    last = torch.empty((B, C), dtype=torch.float32, device=device) if want_state else None
    kept = torch.empty((B, -(-T // NNA_SCAN_KEPT), C), dtype=torch.float32, device=device) if keep else None
    workspace, ws = _scan_workspace(B, T, C, workspace, device, stream)
    _check(lib().nna_gated_scan(*args, t, B, T, C, lp, sp, last.data_ptr() if want_state else None, out.data_ptr(), kept.data_ptr() if keep else None, *ws,
                                device.index, _stream_on(device, stream)))
    if given is not None:
        _written(given)
    result = (out, *((last,) if want_state else ()), *((kept,) if keep else ()))
    return result if len(result) > 1 else out


def nna_gated_scan_backward(gout, kept, x, forget, input=None, lengths=None, gstate=None, want_gstate=False, workspace=None, stream=None):
    """(gx, gforget, ginput or None, gradient of the first state or None): the gradients of a loss through nna_gated_scan, given gout = dLoss/dh (contiguous), what that call
    kept, and gstate = dLoss/d(last state) (None: zero).  `workspace`: nna_gated_scan_workspace bytes (taken here if None)."""
    import torch

    t, (B, T, C), args = _gates(x, forget, input, 3)
    device = x.device
    if stream is not None and (done := _under(stream, device, lambda: nna_gated_scan_backward(gout, kept, x, forget, input, lengths, gstate, want_gstate, workspace))) is not None:
        return done
    lp, gp = _lengths(lengths, B, device), _vector(gstate, "gstate", (B, C), device, none=True)
    kp = _vector(kept, "kept", (B, -(-T // NNA_SCAN_KEPT), C), device)
    if not (isinstance(gout, torch.Tensor) and gout.dtype == x.dtype and gout.is_contiguous() and gout.shape == x.shape and gout.device == device):
        raise TypeError(f"gout must be a contiguous {x.dtype} tensor of shape {(B, T, C)}")
    gx, gf, gi = torch.empty_like(gout), torch.empty_like(gout), None if input is None else torch.empty_like(gout)
    first = torch.empty((B, C), dtype=torch.float32, device=device) if want_gstate else None
    workspace, ws = _scan_workspace(B, T, C, workspace, device, stream)
    _check(lib().nna_gated_scan_backward(gout.data_ptr(), kp, *args, t, B, T, C, lp, gp, gx.data_ptr(), gf.data_ptr(), None if gi is None else gi.data_ptr(),
                                         first.data_ptr() if want_gstate else None, *ws, device.index, _stream_on(device, stream)))
    return gx, gf, gi, first


def nna_gated_scan_step(x, forget, state, input=None, out=None, stream=None):
    """h[B, C] of one new frame x, forget(, input) [B, C] of each sequence; state float32 [B, C] is updated in place."""
    import torch

    t, (B, C), args = _gates(x, forget, input, 2)
    device = x.device
    if stream is not None and (done := _under(stream, device, lambda: nna_gated_scan_step(x, forget, state, input, out))) is not None:
        return done
    sp, given = _vector(state, "state", (B, C), device), out
    if out is None:
        out = x.new_empty((B, C))
    elif not (isinstance(out, torch.Tensor) and out.dtype == x.dtype and out.is_contiguous() and out.shape == x.shape and out.device == device):
        raise TypeError(f"out must be a contiguous {x.dtype} tensor of shape {(B, C)}")
    else:
        _refuse_overlap(out, x, forget, input, state)
    if t == NNA_F32 and any(g is not None and _overlap(state, g) for g in (x, forget, input)):
        raise ValueError("state must not share memory with an input")
    _check(lib().nna_gated_scan_step(*args, t, B, C, sp, out.data_ptr(), device.index, _stream_on(device, stream)))
    _written(state, given)
    return out


_dtype_of = operator.attrgetter("dtype")


def nna_adamw_places(sizes):
    """(where each tensor's states begin, values of all of them together): multiples of 128, in the tensors' order, for tensors of `sizes` values."""
    at = np.zeros(len(sizes) + 1, np.int64)
    np.cumsum([-(-int(n) // NNA_BLOCK8) * NNA_BLOCK8 for n in sizes], out=at[1:])
    return at[:-1], int(at[-1])


def nna_adamw(params, grads, m, v, step, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.01, m_scales=None, v_scales=None, master=None, stream=None):
    """One AdamW step over all of `params`, in place: lists of contiguous float32, bfloat16 or float16 CUDA tensors and their gradients, of their types (None: that tensor and its
    states are left alone).  m, v: the moments, flat, a tensor's beginning at nna_adamw_places' multiple of 128: float32, or int8 (m) and uint8 (v) codes with float32
    m_scales, v_scales [values / 128]; zeros before the first step.  master: flat float32 copies of the 16-bit tensors, likewise, which are updated and rounded from.
    step: the step's number, from 1, of all tensors, or a list of each one's own (tensors whose gradients come and go have taken fewer); step and lr may be CUDA tensors, int64 of one
    value or one for each tensor, and float32 of one value, read when the step runs (so that a graph can record it)."""
    import torch

    tensor, f32 = torch.Tensor, torch.float32
    if not _types:
        _types.update({torch.float32: (NNA_F32, "float32"), torch.bfloat16: (NNA_BF16, "bfloat16"), torch.float16: (NNA_F16, "float16")})
    params, grads = list(params), list(grads)
    if len(params) != len(grads):
        raise ValueError("params and grads must be as many")
    if not (isinstance(m, tensor) and m.is_cuda):
        raise TypeError("m must be a CUDA tensor")
    device = m.device
    # (hundreds of tensors: what is asked of each is asked without a loop in Python, 0.4 us a tensor)
    if any(g is None for g in grads):
        taken = [(p, g) for p, g in zip(params, grads) if g is not None]
        live, live_g = [p for p, _ in taken], [g for _, g in taken]
    else:
        live, live_g = params, grads
    try:
        dtypes = list(map(_dtype_of, params))
        fine = (set(map(tensor.get_device, params)) <= {device.index} and all(map(tensor.is_contiguous, params)) and set(dtypes) <= _types.keys())
        fine_g = fine and (set(map(tensor.get_device, live_g)) <= {device.index} and all(map(tensor.is_contiguous, live_g)) and all(map(tensor.is_same_size, live_g, live))
                           and list(map(_dtype_of, live_g)) == (dtypes if live is params else list(map(_dtype_of, live))))
    except (TypeError, AttributeError, RuntimeError):
        fine = fine_g = False
    if not fine_g:
        raise TypeError(f"params must be contiguous tensors of float32, bfloat16 or float16 on {device}, their gradients of the same types and shapes")
    count = len(params)
    sizes = array.array("q", map(tensor.numel, params))
    size = sum(-(-n // NNA_BLOCK8) for n in sizes) * NNA_BLOCK8
    codes = m_scales is not None or v_scales is not None
    for name, t, dtype, n in (("m", m, torch.int8 if codes else f32, size), ("v", v, torch.uint8 if codes else f32, size),
                              ("m_scales", m_scales, f32, size // NNA_BLOCK8), ("v_scales", v_scales, f32, size // NNA_BLOCK8), ("master", master, f32, size)):
        if t is None and (name == "master" or (name.endswith("scales") and not codes)):
            continue
        if not (isinstance(t, tensor) and t.dtype == dtype and t.device == device and t.is_contiguous() and t.numel() == n):
            raise TypeError(f"{name} must be a contiguous {dtype} tensor of {n} values on {device}")
    step_p = lr_p = steps = None
    apart = 0
    if isinstance(step, tensor):
        if not (step.dtype == torch.int64 and step.device == device and step.is_contiguous() and step.numel() in (1, count)):
            raise TypeError(f"step must be a whole number or one for each tensor, or as many int64 values on {device}")
        step_p, apart = step.data_ptr(), int(step.numel() != 1)
    elif isinstance(step, (list, tuple)):
        if len(step) != count:
            raise ValueError("step must be one number, or one for each tensor")
        steps, apart = array.array("q", step), 1
    else:
        steps = array.array("q", (int(step),))
    if isinstance(lr, tensor):
        if not (lr.dtype == f32 and lr.device == device and lr.numel() == 1):
            raise TypeError(f"lr must be a number, or one float32 value on {device}")
        lr_p, lr = lr.data_ptr(), 0.0
    at = array.array("Q", map(tensor.data_ptr, params))
    at_g = array.array("Q", map(tensor.data_ptr, grads) if live is params else (0 if g is None else g.data_ptr() for g in grads))
    types = array.array("i", [_types[dtypes[0]][0]]) * count if len(set(dtypes)) == 1 else array.array("i", [_types[d][0] for d in dtypes])
    _check(lib().nna_adamw_steps(*(a.buffer_info()[0] if count else None for a in (at, at_g, sizes, types)), count, m.data_ptr(), v.data_ptr(),
                                 *(None if t is None else t.data_ptr() for t in (m_scales, v_scales, master)), size, None if steps is None else steps.buffer_info()[0], step_p, apart,
                                 float(lr), lr_p, float(betas[0]), float(betas[1]), float(eps), float(weight_decay), device.index, _stream_on(device, stream)))
    _all_written([*live, *(t for t in (m, v, m_scales, v_scales, master) if t is not None)])


def nna_adamw_moment(codes, scales, out=None, stream=None):
    """The float32 values that nna_adamw's 8-bit moments stand for: codes int8 (m) or uint8 (v), flat."""
    import torch

    if not (isinstance(codes, torch.Tensor) and codes.is_cuda and codes.dtype in (torch.int8, torch.uint8) and codes.is_contiguous() and codes.numel() % NNA_BLOCK8 == 0):
        raise TypeError("codes must be a contiguous int8 or uint8 CUDA tensor of blocks of 128")
    if stream is not None and (done := _under(stream, codes.device, lambda: nna_adamw_moment(codes, scales, out))) is not None:
        return done
    sp, given = _vector(scales, "scales", (codes.numel() // NNA_BLOCK8,), codes.device), out
    if out is None:
        out = torch.empty_like(codes, dtype=torch.float32)
    elif not (isinstance(out, torch.Tensor) and out.dtype == torch.float32 and out.is_contiguous() and out.shape == codes.shape and out.device == codes.device):
        raise TypeError(f"out must be a contiguous float32 CUDA tensor of shape {tuple(codes.shape)}")
    else:
        _refuse_overlap(out, codes, scales)
    _check(lib().nna_adamw_moment(codes.data_ptr(), codes.dtype == torch.uint8, sp, codes.numel(), out.data_ptr(), codes.device.index, _stream_on(codes.device, stream)))
    if given is not None:
        _written(given)
    return out
