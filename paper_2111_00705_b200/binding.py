"""ctypes binding of libcdadam.so: the same entry points as include/cdadam.h.

Argument marshalling only.  PyTorch supplies device memory and streams; every step of the
method runs in the library's CUDA kernels.  There is no CPU fallback: if the shared library
is missing, loading raises.
"""
import ctypes
import os

import torch

SIGN, TOPK, IDENTITY, RANDK = 0, 1, 2, 3
MARKOV, EF, NAIVE = 0, 1, 2
SERVER = -1
STATE_NAMES = ("ghat_w", "ghat_s", "gtil", "m", "v", "vhat", "x")
OK, ERR_ARG, ERR_ALLOC, ERR_CUDA, ERR_STATE, ERR_TIMEOUT = 0, -1, -2, -3, -4, -5

_LIB_PATH = os.path.join(os.path.dirname(os.path.abspath(__file__)), "libcdadam.so")
_lib = None

_c = ctypes
_SIGNATURES = {
    "cdadam_create": (_c.c_void_p, [_c.c_int64, _c.c_int, _c.c_int, _c.c_int64,
                                    _c.c_float, _c.c_float, _c.c_float, _c.c_float]),
    "cdadam_destroy": (None, [_c.c_void_p]),
    "cdadam_step": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p]),
    "cdadam_step_bf16": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p]),
    "cdadam_step_host": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p]),
    "cdadam_create_shard": (_c.c_void_p, [_c.c_int64, _c.c_int, _c.c_int, _c.c_int, _c.c_int, _c.c_int64,
                                          _c.c_float, _c.c_float, _c.c_float, _c.c_float]),
    "cdadam_step_workers": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p]),
    "cdadam_step_server": (_c.c_int, [_c.c_void_p, _c.c_void_p]),
    "cdadam_step_update": (_c.c_int, [_c.c_void_p, _c.c_void_p]),
    "cdadam_exchange_buffers": (_c.c_int, [_c.c_void_p, _c.POINTER(_c.c_void_p), _c.POINTER(_c.c_void_p),
                                           _c.POINTER(_c.c_void_p), _c.POINTER(_c.c_void_p),
                                           _c.POINTER(_c.c_int64), _c.POINTER(_c.c_int)]),
    "cdadam_create_range": (_c.c_void_p, [_c.c_int64, _c.c_int, _c.c_int64, _c.c_int64, _c.c_int, _c.c_int, _c.c_int,
                                          _c.c_int64, _c.c_float, _c.c_float, _c.c_float, _c.c_float]),
    "cdadam_range_workers": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p]),
    "cdadam_range_server": (_c.c_int, [_c.c_void_p, _c.c_void_p]),
    "cdadam_range_update": (_c.c_int, [_c.c_void_p, _c.c_void_p]),
    "cdadam_range_buffers": (_c.c_int, [_c.c_void_p, _c.POINTER(_c.c_void_p), _c.POINTER(_c.c_void_p),
                                        _c.POINTER(_c.c_int64), _c.POINTER(_c.c_int64), _c.POINTER(_c.c_int),
                                        _c.POINTER(_c.c_void_p)]),
    "cdadam_range_topk": (_c.c_int, [_c.c_void_p, _c.c_int, _c.c_void_p, _c.c_void_p]),
    "cdadam_range_topk_buffer": (_c.c_int, [_c.c_void_p, _c.c_int, _c.POINTER(_c.c_void_p), _c.POINTER(_c.c_int64)]),
    "cdadam_params": (_c.c_void_p, [_c.c_void_p]),
    "cdadam_set_params": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p]),
    "cdadam_set_segments": (_c.c_int, [_c.c_void_p, _c.c_int, _c.POINTER(_c.c_int64)]),
    "cdadam_set_random_sets": (_c.c_int, [_c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p]),
    "cdadam_set_mode": (_c.c_int, [_c.c_void_p, _c.c_int]),
    "cdadam_set_tile": (_c.c_int, [_c.c_void_p, _c.c_int]),
    "cdadam_set_topk_segments": (_c.c_int, [_c.c_void_p, _c.c_int, _c.POINTER(_c.c_int64), _c.POINTER(_c.c_int64)]),
    "cdadam_set_lr": (_c.c_int, [_c.c_void_p, _c.c_float]),
    "cdadam_set_lr_milestones": (_c.c_int, [_c.c_void_p, _c.c_float, _c.c_int, _c.POINTER(_c.c_int64), _c.c_float]),
    "cdadam_set_weight_decay": (_c.c_int, [_c.c_void_p, _c.c_float]),
    "cdadam_get_state": (_c.c_int, [_c.c_void_p, _c.c_int, _c.c_void_p, _c.c_void_p]),
    "cdadam_set_state": (_c.c_int, [_c.c_void_p, _c.c_int, _c.c_void_p, _c.c_void_p]),
    "cdadam_last_payload": (_c.c_int, [_c.c_void_p, _c.c_int, _c.POINTER(_c.c_void_p),
                                       _c.POINTER(_c.c_void_p), _c.POINTER(_c.c_int64)]),
    "cdadam_step_count": (_c.c_int64, [_c.c_void_p]),
    "cdadam_set_step_count": (_c.c_int, [_c.c_void_p, _c.c_int64]),
    "cdadam_device_status": (_c.c_int, [_c.c_void_p, _c.c_void_p]),
    "cdadam_launches_per_step": (_c.c_int, [_c.c_void_p]),
    "cdadam_set_wait_limit": (_c.c_int, [_c.c_void_p, _c.c_int]),
    "cdadam_compress_sign": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int,
                                        _c.POINTER(_c.c_int64), _c.c_void_p, _c.c_void_p,
                                        _c.c_void_p]),
    "cdadam_compress_topk": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_void_p,
                                        _c.c_void_p, _c.c_void_p]),
    "cdadam_compress_sign_static": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p,
                                               _c.c_void_p]),
    "cdadam_set_operator_wait_limit": (_c.c_int, [_c.c_int]),
    "cdadam_layer_norm": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_float,
                                     _c.c_int, _c.c_int, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_void_p]),
    "cdadam_layer_norm_backward": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p,
                                              _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int, _c.c_int, _c.c_int,
                                              _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64,
                                              _c.c_int, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "cdadam_layer_norm_workspace": (_c.c_int64, [_c.c_int64, _c.c_int64, _c.c_int64]),
    "cdadam_token_logprobs": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int, _c.c_int,
                                         _c.c_float, _c.c_int, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p,
                                         _c.c_void_p, _c.c_void_p]),
    "cdadam_token_logprobs_backward": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int,
                                                  _c.c_int, _c.c_float, _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_void_p,
                                                  _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "cdadam_distill": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int,
                                  _c.c_int, _c.c_int, _c.c_float, _c.c_int, _c.c_void_p, _c.c_void_p, _c.c_void_p,
                                  _c.c_int64, _c.c_void_p]),
    "cdadam_rms_norm": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_int64,
                                   _c.c_float, _c.c_int, _c.c_int, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64,
                                   _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64,
                                   _c.c_void_p, _c.c_void_p]),
    "cdadam_rms_norm_backward": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64,
                                            _c.c_void_p, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64,
                                            _c.c_int64, _c.c_int, _c.c_int, _c.c_int, _c.c_void_p, _c.c_int64, _c.c_void_p,
                                            _c.c_int64, _c.c_int, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "cdadam_rms_norm_workspace": (_c.c_int64, [_c.c_int64, _c.c_int64, _c.c_int64]),
    "cdadam_quantize_rows": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int, _c.c_void_p, _c.c_int64,
                                        _c.c_void_p, _c.c_void_p]),
    "cdadam_dequantize_rows": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int,
                                          _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "cdadam_checkpoint8": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int, _c.c_void_p, _c.c_int64,
                                      _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "cdadam_checkpoint8_restore": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_int64, _c.c_int64, _c.c_int64,
                                              _c.c_int, _c.c_void_p, _c.c_int64, _c.c_void_p]),
    "cdadam_matmul8": (_c.c_int, [_c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p, _c.c_int64, _c.c_void_p, _c.c_void_p,
                                  _c.c_int64, _c.c_int64, _c.c_int64, _c.c_int, _c.c_int, _c.c_void_p, _c.c_int64,
                                  _c.c_void_p]),
    "cdadam_profile_enable": (_c.c_int, [_c.c_void_p, _c.c_int]),
    "cdadam_profile_read": (_c.c_int, [_c.c_void_p, _c.POINTER(_c.c_double), _c.POINTER(_c.c_int64)]),
    "cdadam_profile_name": (_c.c_char_p, [_c.c_void_p, _c.c_int]),
    "cdadam_last_error": (_c.c_char_p, []),
}


def exported_symbols():
    """Names of the C entry points this binding expects (those include/cdadam.h declares)."""
    return sorted(_SIGNATURES)


def lib():
    """Load libcdadam.so (once).  Raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError("libcdadam.so is missing: run `python -m paper_2111_00705_b200.build`"
                               " (there is no fallback path)")
        handle = ctypes.CDLL(_LIB_PATH)
        for name, (res, args) in _SIGNATURES.items():
            f = getattr(handle, name)
            f.restype, f.argtypes = res, args
        _lib = handle
    return _lib


class CdadamError(RuntimeError):
    def __init__(self, code, message):
        super().__init__("cdadam error %d: %s" % (code, message))
        self.code = code


def last_error():
    return lib().cdadam_last_error().decode()


def _check(code):
    if code != OK:
        raise CdadamError(code, last_error())


def _stream(stream):
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _dev_f32(t, count, what):
    if not (t.is_cuda and t.dtype == torch.float32 and t.is_contiguous() and t.numel() == count):
        raise ValueError("%s must be a contiguous CUDA float32 tensor of %d elements" % (what, count))
    return ctypes.c_void_p(t.data_ptr())


class _DevView:
    """Zero-copy view of library-owned device memory for torch.as_tensor."""

    def __init__(self, ptr, count, typestr):
        self.__cuda_array_interface__ = {"shape": (count,), "typestr": typestr,
                                         "data": (ptr, False), "version": 2}


def _view(ptr, count, dtype, device):
    typestr = {torch.float32: "<f4", torch.int32: "<i4", torch.float64: "<f8"}[dtype]
    if count == 0:
        return torch.empty(0, dtype=dtype, device=device)
    return torch.as_tensor(_DevView(ptr, count, typestr), device=device)


class CDAdam:
    """One context of the library: n simulated workers and the server on one GPU."""

    def __init__(self, d, n, compressor=SIGN, k=0, beta1=0.9, beta2=0.999, lr=1e-3, eps=1e-8,
                 offsets=None, x0=None, device=None, mode=MARKOV):
        self._h = None
        self.device = torch.device("cuda", torch.cuda.current_device()) if device is None \
            else torch.device(device)
        self.d, self.n, self.compressor, self.k = int(d), int(n), int(compressor), int(k)
        self.q = 1
        self.mode = int(mode)
        self.first_worker, self.n_local = 0, self.n
        with torch.cuda.device(self.device):
            self._h = self._create(beta1, beta2, lr, eps)
        if not self._h:
            raise CdadamError(ERR_ARG, last_error())
        if mode != MARKOV:
            _check(lib().cdadam_set_mode(self._h, int(mode)))
        if offsets is not None:
            self.set_segments(offsets)
        if x0 is not None:
            self.set_params(x0)

    def _create(self, beta1, beta2, lr, eps):
        return lib().cdadam_create(self.d, self.n, self.compressor, self.k, beta1, beta2, lr, eps)

    def close(self):
        if self._h:
            lib().cdadam_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- the three calls of the hot path ------------------------------------------------
    def step(self, grads, stream=None):
        """One iteration of Algorithm 1 on the n x d device gradients."""
        _check(lib().cdadam_step(self._h, _dev_f32(grads, self.n * self.d, "grads"), _stream(stream)))

    def step_bf16(self, grads, stream=None):
        """One iteration on n x d device gradients in bfloat16."""
        if not (grads.is_cuda and grads.dtype == torch.bfloat16 and grads.is_contiguous()
                and grads.numel() == self.n * self.d):
            raise ValueError("grads must be a contiguous CUDA bfloat16 tensor of n*d elements")
        _check(lib().cdadam_step_bf16(self._h, ctypes.c_void_p(grads.data_ptr()), _stream(stream)))

    def step_host(self, grads_host, x_out_host=None, stream=None):
        """The same with host gradients (pinned or pageable) and x copied back to the host."""
        if grads_host.is_cuda or grads_host.dtype != torch.float32 or not grads_host.is_contiguous() \
                or grads_host.numel() != self.n * self.d:
            raise ValueError("grads_host must be a contiguous CPU float32 tensor of n*d elements")
        xo = None
        if x_out_host is not None:
            if x_out_host.is_cuda or x_out_host.dtype != torch.float32 or x_out_host.numel() != self.d \
                    or not x_out_host.is_contiguous():
                raise ValueError("x_out_host must be a contiguous CPU float32 tensor of d elements")
            xo = ctypes.c_void_p(x_out_host.data_ptr())
        _check(lib().cdadam_step_host(self._h, ctypes.c_void_p(grads_host.data_ptr()), xo, _stream(stream)))

    def params(self):
        """The model x as a torch view of the library's memory (no copy)."""
        return _view(lib().cdadam_params(self._h), self.d, torch.float32, self.device)

    # -- helpers ------------------------------------------------------------------------
    def set_params(self, x0, stream=None):
        _check(lib().cdadam_set_params(self._h, _dev_f32(x0, self.d, "x0"), _stream(stream)))

    def set_segments(self, offsets):
        off = (ctypes.c_int64 * len(offsets))(*[int(v) for v in offsets])
        _check(lib().cdadam_set_segments(self._h, len(offsets) - 1, off))
        self.q = len(offsets) - 1

    def set_random_sets(self, workers, server, stream=None):
        """Rand-k: CUDA int32/uint32 tensors with n*k and k increasing coordinates."""
        for t, cnt in ((workers, self.n * self.k), (server, self.k)):
            if not (t.is_cuda and t.is_contiguous() and t.element_size() == 4 and t.numel() == cnt):
                raise ValueError("sets must be contiguous CUDA 32-bit integer tensors of n*k and k elements")
        _check(lib().cdadam_set_random_sets(self._h, ctypes.c_void_p(workers.data_ptr()),
                                            ctypes.c_void_p(server.data_ptr()), _stream(stream)))

    def set_tile(self, tile):
        _check(lib().cdadam_set_tile(self._h, int(tile)))

    def set_topk_segments(self, offsets, k_per_segment):
        """Top-k on every segment on its own; the payload has sum(k_per_segment) entries."""
        off = [int(a) for a in offsets]
        ks = [int(a) for a in k_per_segment]
        if len(ks) != len(off) - 1:
            raise ValueError("one k per segment")
        _check(lib().cdadam_set_topk_segments(self._h, len(ks), (ctypes.c_int64 * len(off))(*off),
                                              (ctypes.c_int64 * len(ks))(*ks)))
        self.k = sum(ks)

    def set_lr(self, lr):
        _check(lib().cdadam_set_lr(self._h, lr))

    def set_lr_milestones(self, base_lr, after_steps, gamma):
        """alpha_t = base_lr * gamma^(number of entries of after_steps that are <= t - 1)."""
        ms = (ctypes.c_int64 * len(after_steps))(*[int(a) for a in after_steps])
        _check(lib().cdadam_set_lr_milestones(self._h, base_lr, len(after_steps), ms, gamma))

    def set_weight_decay(self, weight_decay):
        _check(lib().cdadam_set_weight_decay(self._h, weight_decay))

    def get_state(self, name, stream=None):
        count = self.n_local * self.d if name == "ghat_w" else self.d
        out = torch.empty(count, dtype=torch.float32, device=self.device)
        _check(lib().cdadam_get_state(self._h, STATE_NAMES.index(name), ctypes.c_void_p(out.data_ptr()),
                                      _stream(stream)))
        return out.view(self.n_local, self.d) if name == "ghat_w" else out

    def set_state(self, name, value, stream=None):
        count = self.n_local * self.d if name == "ghat_w" else self.d
        _check(lib().cdadam_set_state(self._h, STATE_NAMES.index(name), _dev_f32(value, count, name),
                                      _stream(stream)))

    def last_payload(self, who):
        """(bits int32[ceil(d/32)], scales float32[q]) or (idx int32[k], val float32[k]) as
        views of library memory, valid until the next step.  Integer words are returned as
        int32 tensors holding the uint32 bit patterns."""
        a, b, cnt = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int64()
        _check(lib().cdadam_last_payload(self._h, who, ctypes.byref(a), ctypes.byref(b), ctypes.byref(cnt)))
        if self.compressor == SIGN:
            return (_view(a.value, (self.d + 31) // 32, torch.int32, self.device),
                    _view(b.value, self.q, torch.float32, self.device))
        return (_view(a.value, self.k, torch.int32, self.device),
                _view(b.value, self.k, torch.float32, self.device))

    def profile_enable(self, on=True):
        _check(lib().cdadam_profile_enable(self._h, 1 if on else 0))

    def profile_read(self):
        """({stage name: total ms}, steps) accumulated since the last read."""
        ms = (ctypes.c_double * 8)()
        steps = ctypes.c_int64()
        _check(lib().cdadam_profile_read(self._h, ms, ctypes.byref(steps)))
        out = {}
        for s in range(8):
            name = lib().cdadam_profile_name(self._h, s).decode()
            if name:
                out[name] = ms[s]
        return out, steps.value

    def device_status(self, stream=None):
        """Wait for the stream; raise if a kernel reported that a bounded wait ran out."""
        _check(lib().cdadam_device_status(self._h, _stream(stream)))

    def set_wait_limit(self, polls):
        """Polls before a kernel's wait on an asynchronous copy gives up (< 0: the default)."""
        _check(lib().cdadam_set_wait_limit(self._h, int(polls)))

    def step_count(self):
        return lib().cdadam_step_count(self._h)

    def set_step_count(self, t):
        """The iteration counter of a run resumed from saved state (see state_dict)."""
        _check(lib().cdadam_set_step_count(self._h, int(t)))

    def state_dict(self, stream=None):
        """Everything a resumed run needs: copies of the seven state vectors and the counter."""
        out = {name: self.get_state(name, stream) for name in STATE_NAMES}
        out["step_count"] = self.step_count()
        return out

    def load_state_dict(self, state, stream=None):
        """Load what state_dict returned into a context created with the same configuration."""
        for name in STATE_NAMES:
            self.set_state(name, state[name].reshape(-1), stream)
        self.set_step_count(state["step_count"])

    def launches_per_step(self):
        return lib().cdadam_launches_per_step(self._h)


class CDAdamShard(CDAdam):
    """A context for the workers [first_worker, first_worker + n_local) of n (scaled sign or
    top-k): one process of a distributed deployment.  An iteration runs in its stages with
    the messages moved by the caller in between (see ``distributed.py``)."""

    def __init__(self, d, n, first_worker, n_local, beta1=0.9, beta2=0.999, lr=1e-3, eps=1e-8,
                 offsets=None, x0=None, device=None, mode=MARKOV, compressor=SIGN, k=0):
        self._shard = (int(first_worker), int(n_local))
        super().__init__(d, n, compressor, k, beta1, beta2, lr, eps, offsets, x0, device, mode)
        self.first_worker, self.n_local = self._shard

    def _create(self, beta1, beta2, lr, eps):
        return lib().cdadam_create_shard(self.d, self.n, self._shard[0], self._shard[1], self.compressor, self.k,
                                         beta1, beta2, lr, eps)

    def step_workers(self, grads, stream=None):
        """Worker stage on the n_local x d device gradients of this context's workers."""
        g = None if self.n_local == 0 else _dev_f32(grads, self.n_local * self.d, "grads")
        _check(lib().cdadam_step_workers(self._h, g, _stream(stream)))

    def step_server(self, stream=None):
        """Server stage from the n worker messages in the exchange buffers."""
        _check(lib().cdadam_step_server(self._h, _stream(stream)))

    def step_update(self, stream=None):
        """gtil += c and the AMSGrad update from the server message in the exchange buffers."""
        _check(lib().cdadam_step_update(self._h, _stream(stream)))

    def exchange_buffers(self):
        """Torch views (no copy) of the message buffers: worker_bits int32[n, words],
        worker_scales float32[n, q], server_bits int32[words], server_scales float32[q].
        worker_scales alternates between two arrays: ask again after every step_workers.
        With top-k the same keys hold the coordinates (int32[n, k], int32[k]) and the values
        (float32[n, k], float32[k]) of the messages."""
        wb, ws, sb, ss = (ctypes.c_void_p() for _ in range(4))
        words, q = ctypes.c_int64(), ctypes.c_int()
        _check(lib().cdadam_exchange_buffers(self._h, ctypes.byref(wb), ctypes.byref(ws), ctypes.byref(sb),
                                             ctypes.byref(ss), ctypes.byref(words), ctypes.byref(q)))
        w, q = words.value, q.value
        return {"worker_bits": _view(wb.value, self.n * w, torch.int32, self.device).view(self.n, w),
                "worker_scales": _view(ws.value, self.n * q, torch.float32, self.device).view(self.n, q),
                "server_bits": _view(sb.value, w, torch.int32, self.device),
                "server_scales": _view(ss.value, q, torch.float32, self.device)}


class CDAdamRange(CDAdam):
    """A context for the coordinates [lo, hi) of a d-dimensional problem with n workers
    (scaled sign): one process of a coordinate-sharded deployment.  Every vector of the
    context has hi - lo coordinates; `offsets` are the segments of the WHOLE problem.  An
    iteration runs in three stages, the l1 sums of the ranges moved by the caller in between
    (see ``distributed.py``)."""

    def __init__(self, d, n, lo, hi, rank, ranks, beta1=0.9, beta2=0.999, lr=1e-3, eps=1e-8,
                 offsets=None, x0=None, device=None, mode=MARKOV, compressor=SIGN, k=0):
        self._range = (int(d), int(lo), int(hi), int(rank), int(ranks))
        self.dim, self.lo, self.hi, self.rank, self.ranks = self._range
        self.q_all = 1 if offsets is None else len(offsets) - 1
        self.k_all = int(k)                 # top-k: entries kept in the whole vector
        super().__init__(hi - lo, n, compressor, min(int(k), hi - lo), beta1, beta2, lr, eps, offsets, x0, device, mode)

    def _create(self, beta1, beta2, lr, eps):
        d, lo, hi, rank, ranks = self._range
        return lib().cdadam_create_range(d, self.n, lo, hi, rank, ranks, self.compressor, self.k_all,
                                         beta1, beta2, lr, eps)

    TOPK_STAGES = 10

    def range_topk(self, stage, grads=None, stream=None):
        """Stage 0..9 of a top-k iteration on the range (0..4 take the n x (hi - lo) gradients)."""
        g = None if grads is None else _dev_f32(grads, self.n * self.d, "grads")
        _check(lib().cdadam_range_topk(self._h, int(stage), g, _stream(stream)))

    def range_topk_buffer(self, stage):
        """The exchange buffer to gather after `stage` as an int32[ranks, words] view, or None."""
        buf, words = ctypes.c_void_p(), ctypes.c_int64()
        _check(lib().cdadam_range_topk_buffer(self._h, int(stage), ctypes.byref(buf), ctypes.byref(words)))
        if not buf.value:
            return None
        return _view(buf.value, self.ranks * words.value, torch.int32, self.device).view(self.ranks, words.value)

    def set_segments(self, offsets):
        super().set_segments(offsets)
        self.q_all = len(offsets) - 1
        self.q = self.range_buffers()["q_local"]

    def range_workers(self, grads, stream=None):
        """Worker pass on the n x (hi - lo) device gradients; writes this range's l1 parts."""
        _check(lib().cdadam_range_workers(self._h, _dev_f32(grads, self.n * self.d, "grads"), _stream(stream)))

    def range_server(self, stream=None):
        """Workers' scales from the gathered parts, server pass on the range, its l1 parts."""
        _check(lib().cdadam_range_server(self._h, _stream(stream)))

    def range_update(self, stream=None):
        """Server's scales from the gathered parts; gtil += c and AMSGrad on the range."""
        _check(lib().cdadam_range_update(self._h, _stream(stream)))

    def range_buffers(self):
        """Torch views (no copy) of the exchange buffers: worker_sums float64[ranks, n, q, 2],
        server_sums float64[ranks, q, 2] (value and rounding error of each range's part of the
        l1 sums; slot [rank] is this context's), q_local and segment_of_local int32[q_local]."""
        ws, ss, seg = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_void_p()
        wd, sd, ql = ctypes.c_int64(), ctypes.c_int64(), ctypes.c_int()
        _check(lib().cdadam_range_buffers(self._h, ctypes.byref(ws), ctypes.byref(ss), ctypes.byref(wd),
                                          ctypes.byref(sd), ctypes.byref(ql), ctypes.byref(seg)))
        q = sd.value // 2
        return {"worker_sums": _view(ws.value, self.ranks * wd.value, torch.float64, self.device).view(self.ranks, self.n, q, 2),
                "server_sums": _view(ss.value, self.ranks * sd.value, torch.float64, self.device).view(self.ranks, q, 2),
                "q_local": ql.value,
                "segment_of_local": _view(seg.value, ql.value, torch.int32, self.device)}


def compress_sign(x, offsets=None, stream=None):
    """Stand-alone scaled-sign compressor on a CUDA vector: (bits int32, scales float32)."""
    d = x.numel()
    q = 1 if offsets is None else len(offsets) - 1
    off = None if offsets is None else (ctypes.c_int64 * len(offsets))(*[int(v) for v in offsets])
    bits = torch.empty((d + 31) // 32, dtype=torch.int32, device=x.device)
    scales = torch.empty(q, dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        _check(lib().cdadam_compress_sign(_dev_f32(x, d, "x"), d, q, off, ctypes.c_void_p(bits.data_ptr()),
                                          ctypes.c_void_p(scales.data_ptr()), _stream(stream)))
    return bits, scales


def compress_topk(x, k, stream=None):
    """Stand-alone top-k compressor on a CUDA vector: (idx int32[k] increasing, val float32[k])."""
    d = x.numel()
    idx = torch.empty(k, dtype=torch.int32, device=x.device)
    val = torch.empty(k, dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        _check(lib().cdadam_compress_topk(_dev_f32(x, d, "x"), d, k, ctypes.c_void_p(idx.data_ptr()),
                                          ctypes.c_void_p(val.data_ptr()), _stream(stream)))
    return idx, val


STATIC_MAX_D = 1 << 28


def compress_sign_static(x, bits=None, scale=None, stream=None):
    """Flat scaled-sign compressor through the entry point that allocates nothing inside the
    library (for callers that cannot allocate device memory at call time).  Pass preallocated
    `bits` (int32[ceil(d/32)]) and `scale` (float32[1]) to keep the whole call free of
    allocations; they are created here only when omitted.  Returns (bits, scale)."""
    d = x.numel()
    if bits is None:
        bits = torch.empty((d + 31) // 32, dtype=torch.int32, device=x.device)
    if scale is None:
        scale = torch.empty(1, dtype=torch.float32, device=x.device)
    with torch.cuda.device(x.device):
        _check(lib().cdadam_compress_sign_static(_dev_f32(x, d, "x"), d, ctypes.c_void_p(bits.data_ptr()),
                                                 ctypes.c_void_p(scale.data_ptr()), _stream(stream)))
    return bits, scale


# -- operators of a worker around its loss ---------------------------------------------------
# They are plain calls: their results have no automatic-differentiation graph, whatever requires_grad
# their inputs have, each gradient is a call of its own, and writing into `out` does not raise a tensor's
# version.  With `stream` a call runs there, and so belongs there what it allocates: other streams have
# to wait for it.
F32, BF16, F16 = 0, 1, 2
MAX_LIST, MAX_VOCAB, MAX_NORM_COLS = 128, 393216, 1048576
_TYPES = {torch.float32: F32, torch.bfloat16: BF16, torch.float16: F16}
_INDEX_TYPES = {torch.int32: 0, torch.int64: 1}


_FLOAT = (torch.float32,)
_raw_stream = torch._C._cuda_getCurrentRawStream if hasattr(torch._C, "_cuda_getCurrentRawStream") else (
    lambda index: torch.cuda.current_stream(index).cuda_stream)
_current = torch._C._cuda_getDevice if hasattr(torch._C, "_cuda_getDevice") else torch.cuda.current_device


def _elsewhere(t, stream):
    """Context of a call that does not run on the current stream of the current device: the
    tensors' device, the given stream.  What the call allocates then belongs to that stream."""
    if not t.is_cuda:
        raise ValueError("the operators take CUDA tensors")
    if stream is None:
        return torch.cuda.device(t.device)
    if stream.device != t.device:
        raise ValueError("the stream belongs to %s, the tensors to %s" % (stream.device, t.device))
    return torch.cuda.stream(stream)


def _matrix(t, what, device=None, shape=None, dtype=None):
    """(pointer, row stride) of a matrix with adjacent row elements."""
    stride = t.stride()
    if len(stride) != 2 or (stride[1] != 1 and t.shape[1] > 1) or t.dtype not in _TYPES:
        raise ValueError("%s must be a matrix of float32, bfloat16 or float16 with adjacent row elements" % what)
    if device is not None and (t.get_device() != device or t.shape != shape or t.dtype != dtype):
        raise ValueError("%s is %s %s on %s, not %s %s on device %d"
                         % (what, tuple(t.shape), t.dtype, t.device, tuple(shape), dtype, device))
    return t.data_ptr(), stride[0]


def _vector(t, what, device, shape, types):
    """Pointer of a contiguous tensor of the given shape and one of the types; None stays None."""
    if t is None:
        return None
    if t.get_device() != device or t.shape != shape or t.dtype not in types or not t.is_contiguous():
        raise ValueError("%s must be a contiguous tensor of shape %s on device %d of one of the types %s"
                         % (what, tuple(shape), device, ", ".join(str(v) for v in types)))
    return t.data_ptr()


def _parameters(weight, bias, cols, device):
    w = _vector(weight, "weight", device, (cols,), _TYPES)
    b = _vector(bias, "bias", device, (cols,), _TYPES)
    if w is not None and b is not None and weight.dtype != bias.dtype:
        raise ValueError("weight and bias differ in type")
    return w, b, _TYPES[weight.dtype] if w is not None else F32 if b is None else _TYPES[bias.dtype]


def set_operator_wait_limit(polls):
    """Polls before the operators' kernels, in this thread's following calls, give up a wait on an
    asynchronous copy (< 0: the default); what depends on the copy is then NaN."""
    _check(lib().cdadam_set_operator_wait_limit(int(polls)))


def layer_norm(x, weight=None, bias=None, eps=1e-5, out=None, stream=None):
    """Layer norm of every row of x (rows x cols): (y, mean, rstd).  weight and bias: cols
    elements of any of the three types (slices of the optimizer's parameter vector, for
    instance).  out: (y, mean, rstd) to write into, each may be None: y is then allocated, mean
    and rstd are not computed.  No automatic differentiation: layer_norm_backward is the gradient."""
    px, sx = _matrix(x, "x")
    device, shape, dtype = x.get_device(), x.shape, x.dtype
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(x, stream):
            return layer_norm(x, weight, bias, eps, out)
    rows, cols = shape
    w, b, wt = _parameters(weight, bias, cols, device)
    if out is None:
        y, mean, rstd = torch.empty(shape, dtype=dtype, device=x.device), *torch.empty(2, rows, device=x.device).unbind(0)
    else:
        y, mean, rstd = out
        if y is None:
            y = torch.empty(shape, dtype=dtype, device=x.device)
    py, sy = _matrix(y, "y", device, shape, dtype)
    code = lib().cdadam_layer_norm(px, sx, w, b, rows, cols, eps, _TYPES[dtype], wt, py, sy,
                                   _vector(mean, "mean", device, (rows,), _FLOAT),
                                   _vector(rstd, "rstd", device, (rows,), _FLOAT), _raw_stream(device))
    if code:
        _check(code)
    return y, mean, rstd


def layer_norm_backward(dy, x, weight, mean, rstd, groups=1, accumulate=False, out=None, workspace=None, stream=None):
    """Gradient of layer_norm: (dx, dweight, dbias), the last two groups x cols, summed over the
    rows of each of `groups` equal parts of the batch (one per worker).  out: the three to write
    into, each may be None: not computed; dweight and dbias may be strided slices of the n x d
    gradient buffer and are added to with accumulate.  workspace: a contiguous CUDA tensor of at
    least layer_norm_workspace(rows, cols, groups) bytes to use instead of allocating one."""
    px, sx = _matrix(x, "x")
    device, shape, dtype = x.get_device(), x.shape, x.dtype
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(x, stream):
            return layer_norm_backward(dy, x, weight, mean, rstd, groups, accumulate, out, workspace)
    rows, cols = shape
    pdy, sdy = _matrix(dy, "dy", device, shape, dtype)
    w, _, wt = _parameters(weight, None, cols, device)
    sums = (groups, cols)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        dx = torch.empty(shape, dtype=dtype, device=x.device)
        dweight, dbias = torch.empty((2,) + sums, device=x.device).unbind(0)
    else:
        dx, dweight, dbias = out
    pdx, sdx = (None, 0) if dx is None else _matrix(dx, "dx", device, shape, dtype)
    some = dweight if dweight is not None else dbias
    gt = None if some is None else some.dtype
    pw, sw = (None, 0) if dweight is None else _matrix(dweight, "dweight", device, sums, gt)
    pb, sb = (None, 0) if dbias is None else _matrix(dbias, "dbias", device, sums, gt)
    if workspace is None:
        need = lib().cdadam_layer_norm_workspace(rows, cols, groups) if some is not None else 0
        workspace = torch.empty(need, dtype=torch.uint8, device=x.device) if need else None
        pws = None if workspace is None else workspace.data_ptr()
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on %s" % x.device)
    else:
        need, pws = workspace.numel() * workspace.element_size(), workspace.data_ptr()
    code = lib().cdadam_layer_norm_backward(
        pdy, sdy, px, sx, w, _vector(mean, "mean", device, (rows,), _FLOAT), _vector(rstd, "rstd", device, (rows,), _FLOAT),
        rows, cols, groups, _TYPES[dtype], wt, F32 if some is None else _TYPES[gt], pdx, sdx, pw, sw, pb, sb,
        1 if accumulate else 0, pws, need, _raw_stream(device))
    if code:
        _check(code)
    return dx, dweight, dbias


def layer_norm_workspace(rows, cols, groups=1):
    """Bytes of workspace layer_norm_backward needs for dweight and dbias."""
    return lib().cdadam_layer_norm_workspace(rows, cols, groups)


def token_logprobs(logits, tokens=None, k=0, temperature=1.0, out=None, stream=None):
    """Per row of logits (rows x vocab): (log probability of tokens[row], entropy, log normaliser,
    the k most probable tokens, their log probabilities), at logits / temperature.  tokens: int32
    or int64, negative = none, or None (the first entry is then None).  out: the five to write
    into, each may be None: not computed.  Ids have the type of tokens (int64 without).  No automatic
    differentiation: token_logprobs_backward is the gradient."""
    pz, sz = _matrix(logits, "logits")
    device, shape = logits.get_device(), logits.shape
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(logits, stream):
            return token_logprobs(logits, tokens, k, temperature, out)
    rows, vocab = shape
    per_row, lists = (rows,), (rows, k)
    pt = _vector(tokens, "tokens", device, per_row, _INDEX_TYPES)
    if out is None:
        logprob, entropy, lse = torch.empty(3, rows, device=logits.device).unbind(0)
        if tokens is None:
            logprob = None
        ids = torch.empty(lists, dtype=torch.int64 if tokens is None else tokens.dtype, device=logits.device)
        top = torch.empty(lists, device=logits.device)
    else:
        logprob, entropy, lse, ids, top = out
    it = tokens if tokens is not None else ids
    if tokens is not None and ids is not None and ids.dtype != tokens.dtype:
        raise ValueError("tokens and ids differ in type")
    code = lib().cdadam_token_logprobs(
        pz, sz, pt, rows, vocab, _TYPES[logits.dtype], 1 if it is None else _INDEX_TYPES.get(it.dtype, -1), temperature, k,
        _vector(logprob, "logprob", device, per_row, _FLOAT), _vector(entropy, "entropy", device, per_row, _FLOAT),
        _vector(lse, "lse", device, per_row, _FLOAT), _vector(ids, "ids", device, lists, _INDEX_TYPES),
        _vector(top, "top", device, lists, _FLOAT), _raw_stream(device))
    if code:
        _check(code)
    return logprob, entropy, lse, ids, top


def token_logprobs_backward(logits, tokens, lse, entropy=None, dlogprob=None, dentropy=None, temperature=1.0, out=None,
                            stream=None):
    """Gradient with respect to the logits of token_logprobs' log probability (dlogprob per row)
    and entropy (dentropy per row), from the forward pass's lse and entropy.  out: where to write
    it (may be logits itself)."""
    pz, sz = _matrix(logits, "logits")
    device, shape, dtype = logits.get_device(), logits.shape, logits.dtype
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(logits, stream):
            return token_logprobs_backward(logits, tokens, lse, entropy, dlogprob, dentropy, temperature, out)
    per_row = (shape[0],)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=logits.device)
    po, so = _matrix(out, "out", device, shape, dtype)
    code = lib().cdadam_token_logprobs_backward(
        pz, sz, _vector(tokens, "tokens", device, per_row, _INDEX_TYPES), shape[0], shape[1], _TYPES[dtype],
        1 if tokens is None else _INDEX_TYPES[tokens.dtype], temperature, _vector(lse, "lse", device, per_row, _FLOAT),
        _vector(entropy, "entropy", device, per_row, _FLOAT), _vector(dlogprob, "dlogprob", device, per_row, _FLOAT),
        _vector(dentropy, "dentropy", device, per_row, _FLOAT), po, so, _raw_stream(device))
    if code:
        _check(code)
    return out


def distill(logits, teacher_ids, teacher_logprobs, dloss=None, temperature=1.0, rest=True, out=None, stream=None):
    """Distillation loss of every row against the teacher's k listed tokens (rows x k, as
    token_logprobs gives them), and with dloss (the gradient of every row's loss) its gradient
    with respect to the logits: (loss, dlogits or None).  rest: the tokens that are not listed
    count as one further outcome; otherwise the list is renormalised.  out: (loss, dlogits) to
    write into, each may be None: not computed.  No automatic differentiation: dlogits is the gradient."""
    pz, sz = _matrix(logits, "logits")
    device, shape, dtype, lists = logits.get_device(), logits.shape, logits.dtype, teacher_ids.shape
    if len(lists) != 2 or lists[0] != shape[0]:
        raise ValueError("teacher_ids has shape %s, not (%d, k)" % (tuple(lists), shape[0]))
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(logits, stream):
            return distill(logits, teacher_ids, teacher_logprobs, dloss, temperature, rest, out)
    per_row = (shape[0],)
    pi = _vector(teacher_ids, "teacher_ids", device, lists, _INDEX_TYPES)
    pq = _vector(teacher_logprobs, "teacher_logprobs", device, lists, _FLOAT)
    if out is None:
        loss = torch.empty(per_row, device=logits.device)
        dz = None if dloss is None else torch.empty(shape, dtype=dtype, device=logits.device)
    else:
        loss, dz = out
    po, so = (None, 0) if dz is None else _matrix(dz, "dlogits", device, shape, dtype)
    code = lib().cdadam_distill(
        pz, sz, pi, pq, shape[0], shape[1], lists[1], _TYPES[dtype], _INDEX_TYPES[teacher_ids.dtype], temperature,
        1 if rest else 0, _vector(dloss, "dloss", device, per_row, _FLOAT), _vector(loss, "loss", device, per_row, _FLOAT),
        po, so, _raw_stream(device))
    if code:
        _check(code)
    return loss, dz


# -- operators in 8 bits ---------------------------------------------------------------------
# Two formats of 8-bit rows, each a pair of tensors: (q int8, scale float32[rows]), a step for every row; and a
# checkpoint (kept int8, exponents uint8[rows, ceil(cols / 32)]), a power of two for every 32 columns.  Those that
# are allocated here have rows that start on 16 bytes, which matmul8 needs.
CHECKPOINT_BLOCK, MAX_INNER = 32, 131071


def _rows8(rows, cols, device):
    return torch.empty(rows, (cols + 15) // 16 * 16, dtype=torch.int8, device=device)[:, :cols]


def _bytes(t, what, device, shape, dtype=torch.int8):
    """(pointer, row stride) of a matrix of bytes."""
    stride = t.stride()
    if t.shape != shape or t.dtype != dtype or t.get_device() != device or (stride[1] != 1 and shape[1] > 1):
        raise ValueError("%s must be %s %s on device %d with adjacent row elements, not %s %s on %s"
                         % (what, tuple(shape), dtype, device, tuple(t.shape), t.dtype, t.device))
    return t.data_ptr(), stride[0]


def _checkpoint(pair, device, shape):
    """(pointer, row stride) of both parts of a checkpoint."""
    kept, exponents = pair
    return _bytes(kept, "kept", device, shape) + _bytes(exponents, "exponents", device, (shape[0], -(-shape[1] // CHECKPOINT_BLOCK)),
                                                        torch.uint8)


def checkpoint8_like(x):
    """A checkpoint (kept, exponents) of a matrix of x's shape to be written into."""
    rows, cols = x.shape
    return _rows8(rows, cols, x.device), torch.empty(rows, -(-cols // CHECKPOINT_BLOCK), dtype=torch.uint8, device=x.device)


def _rms_norm(x, at, device, shape, dtype, weight, residual, eps, y, q, scale, total, rstd, checkpoint):
    px, sx = at
    rows, cols = shape
    pr, sr = (None, 0) if residual is None else _matrix(residual, "residual", device, shape, dtype)
    pt, st = (None, 0) if total is None else _matrix(total, "total", device, shape, dtype)
    py, sy = (None, 0) if y is None else _matrix(y, "y", device, shape, dtype)
    pq, sq = (None, 0) if q is None else _bytes(q, "q", device, shape)
    pk, sk, pe, se = (None, 0, None, 0) if checkpoint is None else _checkpoint(checkpoint, device, shape)
    w = _vector(weight, "weight", device, (cols,), _TYPES)
    code = lib().cdadam_rms_norm(px, sx, pr, sr, w, rows, cols, eps, _TYPES[dtype], F32 if w is None else _TYPES[weight.dtype], pt, st, py, sy, pq, sq,
                                 _vector(scale, "scale", device, (rows,), _FLOAT), pk, sk, pe, se,
                                 _vector(rstd, "rstd", device, (rows,), _FLOAT), _raw_stream(device))
    if code:
        _check(code)


def rms_norm(x, weight=None, residual=None, eps=1e-6, out=None, checkpoint=None, stream=None):
    """Root-mean-square norm of every row of x (rows x cols), or of x + residual where that is given:
    (y, total, rstd), total being the sum as x's type holds it (None without residual).  weight: cols elements of
    any of the three types.  out: (y, total, rstd) to write into, each may be None: y is then allocated, total and
    rstd are not computed.  checkpoint: (kept, exponents) to write the sum's checkpoint into
    (checkpoint8_like).  No automatic differentiation: rms_norm_backward is the gradient."""
    at, device, shape, dtype = _matrix(x, "x"), x.get_device(), x.shape, x.dtype
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(x, stream):
            return rms_norm(x, weight, residual, eps, out, checkpoint)
    if out is None:
        y, rstd = torch.empty(shape, dtype=dtype, device=x.device), torch.empty(shape[0], device=x.device)
        total = None if residual is None else torch.empty_like(y)
    else:
        y, total, rstd = out
        if y is None:
            y = torch.empty(shape, dtype=dtype, device=x.device)
    _rms_norm(x, at, device, shape, dtype, weight, residual, eps, y, None, None, total, rstd, checkpoint)
    return y, total, rstd


def rms_norm8(x, weight=None, residual=None, eps=1e-6, out=None, checkpoint=None, stream=None):
    """rms_norm with its output in 8 bits: (q, scale, total, rstd), as matmul8 takes it.  out: the four to write
    into; total and rstd may be None: not computed."""
    at, device, shape, dtype = _matrix(x, "x"), x.get_device(), x.shape, x.dtype
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(x, stream):
            return rms_norm8(x, weight, residual, eps, out, checkpoint)
    if out is None:
        q = _rows8(*shape, x.device)
        scale, rstd = torch.empty(2, shape[0], device=x.device).unbind(0)
        total = None if residual is None else torch.empty(shape, dtype=dtype, device=x.device)
    else:
        q, scale, total, rstd = out
        if q is None or scale is None:
            raise ValueError("out needs q and scale")
    _rms_norm(x, at, device, shape, dtype, weight, residual, eps, None, q, scale, total, rstd, checkpoint)
    return q, scale, total, rstd


def rms_norm_backward(dy, x, weight, rstd, dtotal=None, groups=1, accumulate=False, out=None, workspace=None, stream=None):
    """Gradient of rms_norm: (dx, dweight).  x: what was normed (the total, or x where there was no residual),
    or its checkpoint (kept, exponents).  dtotal: the gradient that comes along the residual; dx is the gradient of x and
    of the residual alike.  dweight is groups x cols, summed over the rows of each of `groups` equal parts of the
    batch (one per worker).  out: the two to write into, each may be None: not computed; dweight may be a strided slice
    of the n x d gradient buffer and is added to with accumulate.  workspace: a contiguous CUDA tensor of at least
    rms_norm_workspace(rows, cols, groups) bytes to use instead of allocating one."""
    pdy, sdy = _matrix(dy, "dy")
    device, shape, dtype = dy.get_device(), dy.shape, dy.dtype
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(dy, stream):
            return rms_norm_backward(dy, x, weight, rstd, dtotal, groups, accumulate, out, workspace)
    rows, cols = shape
    if isinstance(x, (tuple, list)):
        px, sx, pe, se = _checkpoint(x, device, shape)
    else:
        (px, sx), pe, se = _matrix(x, "x", device, shape, dtype), None, 0
    w = _vector(weight, "weight", device, (cols,), _TYPES)
    wt = F32 if w is None else _TYPES[weight.dtype]
    pdt, sdt = (None, 0) if dtotal is None else _matrix(dtotal, "dtotal", device, shape, dtype)
    sums = (groups, cols)
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs out")
        dx, dweight = torch.empty(shape, dtype=dtype, device=dy.device), torch.empty(sums, device=dy.device)
    else:
        dx, dweight = out
    pdx, sdx = (None, 0) if dx is None else _matrix(dx, "dx", device, shape, dtype)
    gt = None if dweight is None else dweight.dtype
    pw, sw = (None, 0) if dweight is None else _matrix(dweight, "dweight", device, sums, gt)
    if workspace is None:
        need = lib().cdadam_rms_norm_workspace(rows, cols, groups) if dweight is not None else 0
        workspace = torch.empty(need, dtype=torch.uint8, device=dy.device) if need else None
        pws = None if workspace is None else workspace.data_ptr()
    elif workspace.get_device() != device or not workspace.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on %s" % dy.device)
    else:
        need, pws = workspace.numel() * workspace.element_size(), workspace.data_ptr()
    code = lib().cdadam_rms_norm_backward(
        pdy, sdy, px, sx, pe, se, w, _vector(rstd, "rstd", device, (rows,), _FLOAT), pdt, sdt, rows, cols, groups, _TYPES[dtype], wt,
        F32 if gt is None else _TYPES[gt], pdx, sdx, pw, sw, 1 if accumulate else 0, pws, need, _raw_stream(device))
    if code:
        _check(code)
    return dx, dweight


def rms_norm_workspace(rows, cols, groups=1):
    """Bytes of workspace rms_norm_backward needs for dweight."""
    return lib().cdadam_rms_norm_workspace(rows, cols, groups)


def quantize_rows(x, out=None, stream=None):
    """Rows of x in 8 bits, a step for each row: (q, scale).  out: the two to write into."""
    px, sx = _matrix(x, "x")
    device, shape = x.get_device(), x.shape
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(x, stream):
            return quantize_rows(x, out)
    q, scale = (_rows8(*shape, x.device), torch.empty(shape[0], device=x.device)) if out is None else out
    pq, sq = _bytes(q, "q", device, shape)
    code = lib().cdadam_quantize_rows(px, sx, shape[0], shape[1], _TYPES[x.dtype], pq, sq,
                                      _vector(scale, "scale", device, shape[:1], _FLOAT), _raw_stream(device))
    if code:
        _check(code)
    return q, scale


def dequantize_rows(q, scale, dtype=torch.float32, out=None, stream=None):
    """The values q * scale of 8-bit rows, in dtype, or in out and its type."""
    device, shape = q.get_device(), q.shape
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(q, stream):
            return dequantize_rows(q, scale, dtype, out)
    if len(shape) != 2:
        raise ValueError("q must be a matrix")
    pq, sq = _bytes(q, "q", device, shape)
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=q.device)
    po, so = _matrix(out, "out", device, shape, out.dtype)
    code = lib().cdadam_dequantize_rows(pq, sq, _vector(scale, "scale", device, shape[:1], _FLOAT), shape[0], shape[1],
                                        _TYPES[out.dtype], po, so, _raw_stream(device))
    if code:
        _check(code)
    return out


def checkpoint8(x, out=None, stream=None):
    """Checkpoint of x in 8 bits, a power of two for every 32 columns of a row: (kept, exponents).  out: the two to
    write into."""
    px, sx = _matrix(x, "x")
    device, shape = x.get_device(), x.shape
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(x, stream):
            return checkpoint8(x, out)
    out = checkpoint8_like(x) if out is None else out
    code = lib().cdadam_checkpoint8(px, sx, shape[0], shape[1], _TYPES[x.dtype], *_checkpoint(out, device, shape),
                                    _raw_stream(device))
    if code:
        _check(code)
    return tuple(out)


def checkpoint8_restore(kept, exponents, dtype=torch.float32, out=None, stream=None):
    """The values of a checkpoint, in dtype, or in out and its type; exact in the type it was kept from and in
    bfloat16."""
    device, shape = kept.get_device(), kept.shape
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(kept, stream):
            return checkpoint8_restore(kept, exponents, dtype, out)
    if len(shape) != 2:
        raise ValueError("kept must be a matrix")
    if out is None:
        out = torch.empty(shape, dtype=dtype, device=kept.device)
    po, so = _matrix(out, "out", device, shape, out.dtype)
    code = lib().cdadam_checkpoint8_restore(*_checkpoint((kept, exponents), device, shape), shape[0], shape[1],
                                            _TYPES[out.dtype], po, so, _raw_stream(device))
    if code:
        _check(code)
    return out


def matmul8(x, x_scale, w, w_scale, bias=None, dtype=torch.bfloat16, out=None, stream=None):
    """Product of 8-bit rows: y[t, c] = (sum_k x[t, k] w[c, k]) x_scale[t] w_scale[c] + bias[c], tokens x channels in
    dtype, or in out and its type.  x: tokens x inner, w: channels x inner, as rms_norm8 and quantize_rows give them
    (rows start on 16 bytes); bias: channels elements of any of the three types.  There is no gradient."""
    device = x.get_device()
    if device < 0 or stream is not None or device != _current():
        with _elsewhere(x, stream):
            return matmul8(x, x_scale, w, w_scale, bias, dtype, out)
    shape, w_shape = x.shape, w.shape
    if len(shape) != 2 or len(w_shape) != 2:
        raise ValueError("x and w must be matrices")
    (tokens, inner), channels = shape, w_shape[0]
    px, sx = _bytes(x, "x", device, shape)
    pw, sw = _bytes(w, "w", device, (channels, inner))
    pb = _vector(bias, "bias", device, (channels,), _TYPES)
    if out is None:
        out = torch.empty(tokens, channels, dtype=dtype, device=x.device)
    po, so = _matrix(out, "out", device, (tokens, channels), out.dtype)
    code = lib().cdadam_matmul8(
        px, sx, _vector(x_scale, "x_scale", device, (tokens,), _FLOAT), pw, sw, _vector(w_scale, "w_scale", device, (channels,), _FLOAT),
        pb, tokens, channels, inner, _TYPES[out.dtype], F32 if bias is None else _TYPES[bias.dtype], po, so, _raw_stream(device))
    if code:
        _check(code)
    return out
