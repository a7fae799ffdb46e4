"""ctypes binding of libtv.so (C ABI in include/tv.h)."""

import ctypes
import os

HERE = os.path.dirname(os.path.abspath(__file__))

TV_BF16 = 0
TV_FP32 = 1
# tv_create flags: which kernel path a handle uses ("auto" lets the library pick)
PATH_FLAGS = {"auto": 0, "three": 1, "cluster": 2, "persistent": 4}
# tv_create flags: the verification method ("token": the top-down token-level
# verifier the paper compares with; single-kernel paths only)
METHOD_FLAGS = {"traversal": 0, "token": 8}
TV_STATUS = {
    "BAD_TREE": 1,
    "BAD_TOKEN": 2,
    "DUP_SIBLING": 4,
    "ZERO_DRAFT": 8,
    "DEGENERATE": 16,
    "TIMEOUT": 32,
    "BAD_ROW": 64,
    "DRAFT_EXHAUSTED": 128,
    "BAD_SLOT": 256,
    "BAD_MASK": 512,
    "BAD_PAGE": 1024,
    "BAD_LENGTH": 2048,
    "BAD_PATH": 4096,
    "NAN": 8192,
}
# columns (of a weight: and rows) of an 8-bit operand that share a scale
GROUP = 128


class LibraryError(RuntimeError):
    """A call into libtv.so returned an error code."""

    def __init__(self, fn, code, lib):
        msg = lib.tv_strerror(code).decode() if lib is not None else "?"
        super().__init__(f"{fn} failed with code {code}: {msg}")
        self.code = code


def library_path():
    return os.path.join(HERE, "libtv.so")


_LIB = None

_P = ctypes.c_void_p
_I = ctypes.c_int
_F = ctypes.c_float


class _Context(ctypes.Structure):
    """tv_context of include/tv.h."""
    _fields_ = [("slots", ctypes.c_int32), ("counts", _P), ("bias", _P), ("marks", _P)]


class _Cache(ctypes.Structure):
    """tv_cache of include/tv.h."""
    _fields_ = [("layers", ctypes.c_int32), ("pages", ctypes.c_int32),
                ("kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("page_size", ctypes.c_int32), ("data", _P), ("exponents", _P)]


_SIGS = {
    "tv_create": (_I, [ctypes.POINTER(_P), _I, _I, _I, _I, _I, ctypes.c_uint]),
    "tv_verify_batch": (_I, [_P, _I, _I, _P, _P, _P, _P, _F, _P, _P, _P, _P, _P]),
    "tv_verify_batch_debug": (_I, [_P, _I, _I, _P, _P, _P, _P, _F, _P, _P, _P, _P, _P, _P, _P,
                                   _P]),
    "tv_verify_batch_host": (_I, [_P, _I, _I, _P, _P, _P, _P, _F, _P, _P, _P, _P, _P]),
    "tv_verify_batch_stats": (_I, [_P, _I, _I, _P, _P, _P, _P, _F, _P, _P, _P, _P, _P, _P, _P,
                                   _P]),
    "tv_lm_head": (_I, [_P, _I, _I, _P, _P, _F, _P, _P, _P]),
    "tv_draft_children": (_I, [_P, _I, _I, _P, _P, _P, _P, _P]),
    "tv_rms_norm": (_I, [_P, _I, _I, _I, _P, _P, _I, _P, _F, _P, _P, _P, _P]),
    "tv_quantize_weight": (_I, [_P, _I, _I, _I, _P, _P, _P, _P]),
    "tv_lm_head_scaled": (_I, [_P, _I, _I, _P, _P, _P, _P, _F, _P, _P, _P]),
    "tv_context_clear": (_I, [_P, _P, _I, _P, _P]),
    "tv_context_add": (_I, [_P, _P, _I, _I, _I, _P, _P, _P, _P]),
    "tv_context_accept": (_I, [_P, _P, _I, _I, _P, _P, _P, _P, _P]),
    "tv_process_logits": (_I, [_P, _P, _I, _I, _P, _P, _P, _P, _P, _P, _I, _F, _P, _P, _P, _P]),
    "tv_cache_write": (_I, [_P, _P, _I, _I, _I, _I, _P, _P, _P, _P, _I, _P, _P]),
    "tv_cache_read": (_I, [_P, _P, _I, _I, _I, _I, _P, _P, _I, _P, _P, _P, _P]),
    "tv_cache_accept": (_I, [_P, _P, _I, _I, _P, _P, _I, _P, _P, _P, _P]),
    "tv_tree_attention": (_I, [_P, _P, _I, _I, _I, _I, _P, _P, _P, _I, _P, _P, _F, _P, _P]),
    "tv_last_host_copy_bytes": (_I, [_P, _P, _P]),
    "tv_get_status": (_I, [_P, ctypes.POINTER(ctypes.c_uint32)]),
    "tv_debug_withhold_job": (_I, [_P, _I]),
    "tv_destroy": (_I, [_P]),
    "tv_set_phase_timing": (_I, [_P, _I]),
    "tv_last_phase_ms": (_I, [_P, ctypes.POINTER(ctypes.c_float)]),
    "tv_launch_shape": (_I, [_P, _I, _I, ctypes.POINTER(_I), ctypes.POINTER(_I),
                             ctypes.POINTER(_I), ctypes.POINTER(_I)]),
    "tv_verify_batch_noalloc": (_I, [_I, _I, _I, _I, _I, _P, _P, _P, _P, _F, _P, _P, _P, _P,
                                     _P]),
    "tv_strerror": (ctypes.c_char_p, [_I]),
    "tv_version": (_I, []),
}


def library():
    """Load libtv.so (raises if it has not been built: there is no fallback)."""
    global _LIB
    if _LIB is None:
        path = library_path()
        if not os.path.exists(path):
            raise ImportError(
                f"{path} is missing: build it with `python -m paper_2505_12398_gb300.build` "
                "(or __graft_entry__.build()); the verifier has no CPU implementation")
        lib = ctypes.CDLL(path)
        for name, (res, args) in _SIGS.items():
            fn = getattr(lib, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = lib
    return _LIB


def status_names(bits):
    return [k for k, v in TV_STATUS.items() if bits & v]


def _ptr(t):
    return ctypes.c_void_p(t.data_ptr()) if t is not None else ctypes.c_void_p(0)


def _stream_ptr(stream):
    import torch
    if stream is None:
        stream = torch.cuda.current_stream()
    return ctypes.c_void_p(stream.cuda_stream)


def _check_out(t, dtype, shape, device):
    """An output tensor the library writes: its dtype, shape, contiguity and
    device must be what the call's sizes say (the kernels trust them)."""
    if t.dtype != dtype or tuple(t.shape) != tuple(shape) or not t.is_contiguous() \
            or t.device != device:
        raise ValueError(f"output: expected a contiguous {dtype} {tuple(shape)} tensor on "
                         f"{device}, got {t.dtype} {tuple(t.shape)} on {t.device}")


def _check_in(t, dtype, shape, device, name):
    if t.dtype != dtype or t.shape != shape or not t.is_contiguous() or t.device != device:
        raise ValueError(f"{name}: expected a contiguous {dtype} {shape} tensor on {device}, "
                         f"got {t.dtype} {tuple(t.shape)} on {t.device}")


def _at(t):
    """A tensor's address as an argument of the library (0 for None)."""
    return 0 if t is None else t.data_ptr()


def _raw_stream(index):
    """The current stream of a device as a cudaStream_t, without the object that
    torch.cuda.current_stream builds (3 us of a small call's 13)."""
    import torch
    get = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return get(index) if get is not None else torch.cuda.current_stream(index).cuda_stream


class Verifier:
    """Owns a ``tv_handle`` (device workspace) for one device and size limits.

    All tensors passed to :meth:`verify` must be contiguous CUDA tensors on
    the handle's device with the dtypes and layouts of include/tv.h.
    """

    def __init__(self, vocab, max_nodes, max_batch, logit_dtype="bf16", device=0, path="auto",
                 method="traversal"):
        import torch
        self.lib = library()
        if logit_dtype in ("bf16", torch.bfloat16, TV_BF16):
            self.dtype_code, self.logit_dtype = TV_BF16, torch.bfloat16
        elif logit_dtype in ("fp32", torch.float32, TV_FP32):
            self.dtype_code, self.logit_dtype = TV_FP32, torch.float32
        else:
            raise ValueError(f"unsupported logit dtype {logit_dtype}")
        self.vocab, self.max_nodes, self.max_batch = vocab, max_nodes, max_batch
        self.device = torch.device("cuda", device) if isinstance(device, int) else torch.device(device)
        h = ctypes.c_void_p()
        if path not in PATH_FLAGS:
            raise ValueError(f"unknown path {path!r}; one of {sorted(PATH_FLAGS)}")
        if method not in METHOD_FLAGS:
            raise ValueError(f"unknown method {method!r}; one of {sorted(METHOD_FLAGS)}")
        self.method = method
        rc = self.lib.tv_create(ctypes.byref(h), self.device.index or 0, vocab, max_nodes,
                                max_batch, self.dtype_code,
                                PATH_FLAGS[path] | METHOD_FLAGS[method])
        if rc != 0:
            raise LibraryError("tv_create", rc, self.lib)
        self.handle = h

    def close(self):
        if getattr(self, "handle", None) is not None and self.handle.value:
            self.lib.tv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, parents, tokens, logits, drafts, uniforms):
        import torch
        B, R = parents.shape
        N = R - 1
        V = self.vocab
        exp = [(parents, torch.int32, (B, R)), (tokens, torch.int32, (B, R)),
               (logits, self.logit_dtype, (B, R, V)), (drafts, torch.float32, (B, R, V)),
               (uniforms, torch.float32, (B, R + 1))]
        for t, dt, shape in exp:
            if t.dtype != dt or tuple(t.shape) != shape:
                raise ValueError(f"expected {dt} {shape}, got {t.dtype} {tuple(t.shape)}")
            if not t.is_contiguous():
                raise ValueError("tensors must be contiguous")
            if t.device != self.device:
                raise ValueError(f"tensor on {t.device}, handle on {self.device}")
        return B, N

    def verify(self, parents, tokens, logits, drafts, temperature, uniforms,
               out=None, stream=None, debug=False, margins=False):
        """Returns (path [B,N] int32, tau [B] int32, bonus [B] int32) as CUDA
        tensors, plus (node_p [B,N+1] f32, stats [B,5] int32) when ``debug``,
        plus margins [B,2] f32 (test, bonus) when ``margins`` too.
        Asynchronous on ``stream`` (default: torch's current stream)."""
        import torch
        B, N = self._check(parents, tokens, logits, drafts, uniforms)
        if out is None:
            path = torch.empty(B, N, dtype=torch.int32, device=self.device)
            tau = torch.empty(B, dtype=torch.int32, device=self.device)
            bonus = torch.empty(B, dtype=torch.int32, device=self.device)
        else:
            path, tau, bonus = out
            for t, shape in ((path, (B, N)), (tau, (B,)), (bonus, (B,))):
                _check_out(t, torch.int32, shape, self.device)
        sp = _stream_ptr(stream)
        if debug:
            node_p = torch.empty(B, N + 1, dtype=torch.float32, device=self.device)
            stats = torch.empty(B, 5, dtype=torch.int32, device=self.device)
            margin = torch.empty(B, 2, dtype=torch.float32, device=self.device)
            rc = self.lib.tv_verify_batch_debug(
                self.handle, B, N, _ptr(parents), _ptr(tokens), _ptr(logits), _ptr(drafts),
                float(temperature), _ptr(uniforms), _ptr(path), _ptr(tau), _ptr(bonus),
                _ptr(node_p), _ptr(stats), _ptr(margin), sp)
            if rc != 0:
                raise LibraryError("tv_verify_batch_debug", rc, self.lib)
            if margins:
                return path, tau, bonus, node_p, stats, margin
            return path, tau, bonus, node_p, stats
        rc = self.lib.tv_verify_batch(
            self.handle, B, N, _ptr(parents), _ptr(tokens), _ptr(logits), _ptr(drafts),
            float(temperature), _ptr(uniforms), _ptr(path), _ptr(tau), _ptr(bonus), sp)
        if rc != 0:
            raise LibraryError("tv_verify_batch", rc, self.lib)
        return path, tau, bonus

    def lm_head(self, hidden, weight, temperature, out=None, stream=None):
        """Logits [M, V] bf16 = hidden [M, K] x weight [V, K]^T on the tensor
        cores, and each row's normaliser [M, 2] fp32 (max, sum of
        2^((l - max) log2(e) / T)) of the stored logits (tv_lm_head).
        ``out`` = (logits, row_stats) to write into given tensors."""
        import torch
        M, K = hidden.shape
        for t, shape in ((hidden, (M, K)), (weight, (self.vocab, K))):
            if t.dtype != torch.bfloat16 or tuple(t.shape) != shape or not t.is_contiguous() \
                    or t.device != self.device:
                raise ValueError(f"expected a contiguous bf16 {shape} tensor on {self.device}")
        if out is None:
            logits = torch.empty(M, self.vocab, dtype=torch.bfloat16, device=self.device)
            row_stats = torch.empty(M, 2, dtype=torch.float32, device=self.device)
        else:
            logits, row_stats = out
            if logits.numel() != M * self.vocab or row_stats.numel() != 2 * M:
                raise ValueError("output: logits must hold M x V and row_stats M x 2 values")
            _check_out(logits, torch.bfloat16, logits.shape, self.device)
            _check_out(row_stats, torch.float32, row_stats.shape, self.device)
        rc = self.lib.tv_lm_head(self.handle, M, K, _ptr(hidden), _ptr(weight),
                                 float(temperature), _ptr(logits), _ptr(row_stats),
                                 _stream_ptr(stream))
        if rc != 0:
            raise LibraryError("tv_lm_head", rc, self.lib)
        return logits, row_stats

    def draft_children(self, parents, drafts, uniforms, out=None, stream=None):
        """Tokens [B, N+1] int32 of every node, drawn from its parent's draft
        row without its earlier siblings' tokens (Definition 1), node c with
        uniforms[:, c] (tv_draft_children).  parents [B, N+1] int32, drafts
        [B, N+1, V] fp32, uniforms [B, N+1] fp32, all on the handle's device."""
        import torch
        B, R = parents.shape
        for t, dt, shape in ((parents, torch.int32, (B, R)), (drafts, torch.float32, (B, R, self.vocab)),
                             (uniforms, torch.float32, (B, R))):
            if t.dtype != dt or tuple(t.shape) != shape or not t.is_contiguous() \
                    or t.device != self.device:
                raise ValueError(f"expected a contiguous {dt} {shape} tensor on {self.device}")
        tokens = torch.empty(B, R, dtype=torch.int32, device=self.device) if out is None else out
        _check_out(tokens, torch.int32, (B, R), self.device)
        rc = self.lib.tv_draft_children(self.handle, B, R - 1, _ptr(parents), _ptr(drafts),
                                        _ptr(uniforms), _ptr(tokens), _stream_ptr(stream))
        if rc != 0:
            raise LibraryError("tv_draft_children", rc, self.lib)
        return tokens

    def _stream(self, stream):
        return _raw_stream(self.device.index or 0) if stream is None else stream.cuda_stream

    def _empty(self, stream, *outputs):
        """New outputs ((shape, dtype) or None each), of the stream that writes them: memory
        of another stream's might still be in use there."""
        import torch
        if stream is not None:
            with torch.cuda.stream(stream):
                return self._empty(None, *outputs)
        empty, dev = torch.empty, self.device
        return [empty(o[0], dtype=o[1], device=dev) if o is not None else None for o in outputs]

    def _float_code(self, t, name):
        import torch
        if t.dtype == torch.bfloat16:
            return TV_BF16
        if t.dtype == torch.float32:
            return TV_FP32
        raise ValueError(f"{name}: expected a bf16 or float32 tensor, got {t.dtype}")

    def rms_norm(self, x, weight, residual=None, eps=1e-5, quantize=True, out=None, stream=None):
        """Root-mean-square norm of the rows of x + residual (tv_rms_norm).
        x, residual [M, K] bf16 or fp32 of one type, weight [K] bf16 or fp32.
        Returns (values e4m3 [M, K], scales fp32 [M, ceil(K / 128)], residual) with
        ``quantize``, else (values bf16 [M, K], residual); the last is x + residual in
        x's type, None without a residual.  ``out`` gives the same tuple to write into
        (its residual may be x or residual itself)."""
        import torch
        M, K = x.shape
        code, wcode = self._float_code(x, "x"), self._float_code(weight, "weight")
        _check_in(x, x.dtype, (M, K), self.device, "x")
        _check_in(weight, weight.dtype, (K,), self.device, "weight")
        if residual is not None:
            _check_in(residual, x.dtype, (M, K), self.device, "residual")
        kind = torch.float8_e4m3fn if quantize else torch.bfloat16
        groups = (K + GROUP - 1) // GROUP
        if out is None:
            y, scales, total = self._empty(
                stream, ((M, K), kind), ((M, groups), torch.float32) if quantize else None,
                ((M, K), x.dtype) if residual is not None else None)
        else:
            y, scales, total = out if quantize else (out[0], None, out[1])
            _check_out(y, kind, (M, K), self.device)
            if quantize:
                _check_out(scales, torch.float32, (M, groups), self.device)
            if (total is None) != (residual is None):
                raise ValueError("output: a residual is written where one is given")
            if total is not None:
                _check_out(total, x.dtype, (M, K), self.device)
        rc = self.lib.tv_rms_norm(self.handle, M, K, code, _at(x), _at(residual), wcode,
                                  _at(weight), float(eps), _at(total), _at(y), _at(scales),
                                  self._stream(stream))
        if rc != 0:
            raise LibraryError("tv_rms_norm", rc, self.lib)
        return (y, scales, total) if quantize else (y, total)

    def quantize_weight(self, weight, out=None, stream=None):
        """(values e4m3 [rows, K], scales fp32 [ceil(rows / 128), ceil(K / 128)]) of a bf16
        or fp32 weight [rows, K], one scale per 128 x 128 block (tv_quantize_weight)."""
        import torch
        rows, K = weight.shape
        code = self._float_code(weight, "weight")
        _check_in(weight, weight.dtype, (rows, K), self.device, "weight")
        blocks = ((rows + GROUP - 1) // GROUP, (K + GROUP - 1) // GROUP)
        if out is None:
            q, scales = self._empty(stream, ((rows, K), torch.float8_e4m3fn),
                                    (blocks, torch.float32))
        else:
            q, scales = out
            _check_out(q, torch.float8_e4m3fn, (rows, K), self.device)
            _check_out(scales, torch.float32, blocks, self.device)
        rc = self.lib.tv_quantize_weight(self.handle, rows, K, code, _at(weight), _at(q),
                                         _at(scales), self._stream(stream))
        if rc != 0:
            raise LibraryError("tv_quantize_weight", rc, self.lib)
        return q, scales

    def lm_head_fp8(self, hidden, hidden_scales, weight, weight_scales, temperature=None,
                    out=None, stream=None):
        """lm_head() on e4m3 operands with block scales (tv_lm_head_scaled): hidden [M, K] with
        scales [M, ceil(K / 128)] (rms_norm), weight [V, K] with scales
        [ceil(V / 128), ceil(K / 128)] (quantize_weight).  Returns (logits [M, V] bf16,
        row_stats [M, 2] fp32); without a temperature the latter is None and not
        computed.  ``out`` = (logits, row_stats)."""
        import torch
        M, K = hidden.shape
        V, groups = self.vocab, (K + GROUP - 1) // GROUP
        _check_in(hidden, torch.float8_e4m3fn, (M, K), self.device, "hidden")
        _check_in(hidden_scales, torch.float32, (M, groups), self.device, "hidden_scales")
        _check_in(weight, torch.float8_e4m3fn, (V, K), self.device, "weight")
        _check_in(weight_scales, torch.float32, ((V + GROUP - 1) // GROUP, groups), self.device,
                  "weight_scales")
        if out is None:
            logits, row_stats = self._empty(
                stream, ((M, V), torch.bfloat16),
                ((M, 2), torch.float32) if temperature is not None else None)
        else:
            logits, row_stats = out
            _check_out(logits, torch.bfloat16, (M, V), self.device)
            if (row_stats is None) != (temperature is None):
                raise ValueError("output: row_stats are written where a temperature is given")
            if row_stats is not None:
                _check_out(row_stats, torch.float32, (M, 2), self.device)
        rc = self.lib.tv_lm_head_scaled(
            self.handle, M, K, _at(hidden), _at(hidden_scales), _at(weight),
            _at(weight_scales), float(temperature) if temperature is not None else 0.0,
            _at(logits), _at(row_stats), self._stream(stream))
        if rc != 0:
            raise LibraryError("tv_lm_head_scaled", rc, self.lib)
        return logits, row_stats

    def process_logits(self, context, parents, tokens, logits, temperature, slots=None,
                       penalties=None, masks=None, mask_index=None, out=None, stream=None):
        """Penalties, biases and grammar masks on the logits of every tree row, and the
        rows' normalisers after them (tv_process_logits).  context: a TokenContext or
        None; parents, tokens [B, N+1] int32; logits [B, N+1, V]; slots [B] int32 (None:
        request b is slot b); penalties [B, 3] fp32 (repetition, frequency, presence);
        masks [n, ceil(V / 32)] int32 (a set bit allows the token) with mask_index
        [B, N+1] int32 (-1: none).  Returns (logits [B, N+1, V], row_stats [B, N+1, 2]
        fp32), which verify_stats() takes; ``out`` the same to write into (its logits may
        be ``logits``)."""
        import torch
        B, R = parents.shape
        V = self.vocab
        _check_in(parents, torch.int32, (B, R), self.device, "parents")
        _check_in(tokens, torch.int32, (B, R), self.device, "tokens")
        _check_in(logits, self.logit_dtype, (B, R, V), self.device, "logits")
        if slots is not None:
            _check_in(slots, torch.int32, (B,), self.device, "slots")
        if penalties is not None:
            _check_in(penalties, torch.float32, (B, 3), self.device, "penalties")
        n_masks = 0
        if (masks is None) != (mask_index is None):
            raise ValueError("masks and mask_index go together")
        if masks is not None:
            n_masks = masks.shape[0]
            _check_in(masks, torch.int32, (n_masks, (V + 31) // 32), self.device, "masks")
            _check_in(mask_index, torch.int32, (B, R), self.device, "mask_index")
        if context is not None and (context.vocab != V or context.device != self.device):
            raise ValueError("the context is for another vocabulary or device")
        if out is None:
            res, row_stats = self._empty(stream, ((B, R, V), self.logit_dtype),
                                         ((B, R, 2), torch.float32))
        else:
            res, row_stats = out
            _check_out(res, self.logit_dtype, (B, R, V), self.device)
            _check_out(row_stats, torch.float32, (B, R, 2), self.device)
        rc = self.lib.tv_process_logits(
            self.handle, context.ref if context is not None else None, B, R - 1, _at(slots),
            _at(parents), _at(tokens), _at(penalties), _at(masks), _at(mask_index), n_masks,
            float(temperature), _at(logits), _at(res), _at(row_stats), self._stream(stream))
        if rc != 0:
            raise LibraryError("tv_process_logits", rc, self.lib)
        return res, row_stats

    def verify_stats(self, parents, tokens, logits, drafts, temperature, uniforms, row_stats,
                     out=None, stream=None, debug=False):
        """verify() with the rows' normalisers given ([B, N+1, 2] or [B*(N+1), 2]
        fp32, e.g. from lm_head) (tv_verify_batch_stats)."""
        import torch
        B, N = self._check(parents, tokens, logits, drafts, uniforms)
        if row_stats.dtype != torch.float32 or row_stats.numel() != 2 * B * (N + 1) or \
                not row_stats.is_contiguous() or row_stats.device != self.device:
            raise ValueError("row_stats must be a contiguous float32 [B*(N+1), 2] tensor "
                             "on the handle's device")
        if out is None:
            path = torch.empty(B, N, dtype=torch.int32, device=self.device)
            tau = torch.empty(B, dtype=torch.int32, device=self.device)
            bonus = torch.empty(B, dtype=torch.int32, device=self.device)
        else:
            path, tau, bonus = out
            for t, shape in ((path, (B, N)), (tau, (B,)), (bonus, (B,))):
                _check_out(t, torch.int32, shape, self.device)
        node_p = torch.empty(B, N + 1, dtype=torch.float32, device=self.device) if debug else None
        stats = torch.empty(B, 5, dtype=torch.int32, device=self.device) if debug else None
        rc = self.lib.tv_verify_batch_stats(
            self.handle, B, N, _ptr(parents), _ptr(tokens), _ptr(logits), _ptr(drafts),
            float(temperature), _ptr(uniforms), _ptr(row_stats), _ptr(path), _ptr(tau),
            _ptr(bonus), _ptr(node_p), _ptr(stats), _stream_ptr(stream))
        if rc != 0:
            raise LibraryError("tv_verify_batch_stats", rc, self.lib)
        return (path, tau, bonus, node_p, stats) if debug else (path, tau, bonus)

    def verify_host(self, parents, tokens, logits, drafts, temperature, uniforms,
                    out, stream=None):
        """Same verification from host (CPU, ideally pinned) tensors; copies in,
        verifies, copies the outputs into ``out`` = (path, tau, bonus) host
        tensors and synchronises."""
        B, R = parents.shape
        N = R - 1
        path, tau, bonus = out
        rc = self.lib.tv_verify_batch_host(
            self.handle, B, N, _ptr(parents), _ptr(tokens), _ptr(logits), _ptr(drafts),
            float(temperature), _ptr(uniforms), _ptr(path), _ptr(tau), _ptr(bonus),
            _stream_ptr(stream))
        if rc != 0:
            raise LibraryError("tv_verify_batch_host", rc, self.lib)
        return path, tau, bonus

    def last_host_copy_bytes(self):
        """(host-to-device, device-to-host) bytes of the last verify_host call
        (tv_last_host_copy_bytes)."""
        h2d, d2h = ctypes.c_uint64(), ctypes.c_uint64()
        rc = self.lib.tv_last_host_copy_bytes(self.handle, ctypes.byref(h2d), ctypes.byref(d2h))
        if rc != 0:
            raise LibraryError("tv_last_host_copy_bytes", rc, self.lib)
        return h2d.value, d2h.value

    def set_phase_timing(self, enable=True):
        rc = self.lib.tv_set_phase_timing(self.handle, 1 if enable else 0)
        if rc != 0:
            raise LibraryError("tv_set_phase_timing", rc, self.lib)

    def last_phase_ms(self):
        """Device milliseconds of (prep, row normalisers, traversal) of the
        last call made with phase timing on (waits for it)."""
        ms = (ctypes.c_float * 3)()
        rc = self.lib.tv_last_phase_ms(self.handle, ms)
        if rc != 0:
            raise LibraryError("tv_last_phase_ms", rc, self.lib)
        return [float(x) for x in ms]

    def launch_shape(self, B, N):
        """(path code, CTAs per tree, consumer warps per CTA, ring stages);
        path code 0 = two kernels, 1 = cluster per tree, 2 = persistent."""
        out = [ctypes.c_int() for _ in range(4)]
        rc = self.lib.tv_launch_shape(self.handle, B, N, *[ctypes.byref(o) for o in out])
        if rc != 0:
            raise LibraryError("tv_launch_shape", rc, self.lib)
        return tuple(o.value for o in out)

    def withhold_job(self, tree):
        """Test hook (tv_debug_withhold_job): the next persistent-kernel call
        never publishes tree ``tree``'s first job, so its waits run out."""
        rc = self.lib.tv_debug_withhold_job(self.handle, int(tree))
        if rc != 0:
            raise LibraryError("tv_debug_withhold_job", rc, self.lib)

    def status(self):
        """Synchronise and return (and clear) the TV_STATUS_* bits raised."""
        v = ctypes.c_uint32(0)
        rc = self.lib.tv_get_status(self.handle, ctypes.byref(v))
        if rc != 0:
            raise LibraryError("tv_get_status", rc, self.lib)
        return v.value


class TokenContext:
    """What the texts of up to ``slots`` requests add up to (tv_context): per slot and
    token the count of generated occurrences and a prompt bit (``counts`` [slots, V]
    int32: count << 1 | prompt), a bias (``bias`` [slots, V] fp32) and a bit in ``marks``
    [slots, ceil(V / 32)] int32 for every token that has any.  Empty when created
    without arrays.  Its updates run on the given (default: current) stream."""

    def __init__(self, verifier, slots, counts=None, bias=None, marks=None):
        import torch
        self.verifier, self.slots = verifier, slots
        self.vocab, self.device = verifier.vocab, verifier.device
        V, dev = self.vocab, self.device
        words = (V + 31) // 32
        self.counts = torch.zeros(slots, V, dtype=torch.int32, device=dev) \
            if counts is None else counts
        self.bias = torch.zeros(slots, V, dtype=torch.float32, device=dev) if bias is None \
            else bias
        self.marks = torch.zeros(slots, words, dtype=torch.int32, device=dev) if marks is None \
            else marks
        _check_in(self.counts, torch.int32, (slots, V), dev, "counts")
        _check_in(self.bias, torch.float32, (slots, V), dev, "bias")
        _check_in(self.marks, torch.int32, (slots, words), dev, "marks")
        self.struct = _Context(slots, self.counts.data_ptr(), self.bias.data_ptr(),
                               self.marks.data_ptr())
        self.ref = ctypes.cast(ctypes.pointer(self.struct), _P)

    def _slots(self, slots, B):
        import torch
        if slots is not None:
            _check_in(slots, torch.int32, (B,), self.device, "slots")
        return _at(slots)

    def _call(self, name, *args):
        rc = getattr(self.verifier.lib, name)(self.verifier.handle, self.ref, *args)
        if rc != 0:
            raise LibraryError(name, rc, self.verifier.lib)

    def clear(self, slots, stream=None):
        """Empties the given slots ([n] int32, distinct)."""
        self._call("tv_context_clear", slots.numel(), self._slots(slots, slots.numel()),
                   self.verifier._stream(stream))

    def _add(self, kind, tokens, values, slots, stream):
        import torch
        B, n = tokens.shape
        _check_in(tokens, torch.int32, (B, n), self.device, "tokens")
        if values is not None:
            _check_in(values, torch.float32, (B, n), self.device, "values")
        self._call("tv_context_add", kind, B, n, self._slots(slots, B), _at(tokens),
                   _at(values), self.verifier._stream(stream))

    def add_prompt(self, tokens, slots=None, stream=None):
        """Prompt tokens [B, n] int32 of B requests; negative entries are skipped."""
        self._add(0, tokens, None, slots, stream)

    def add_generated(self, tokens, slots=None, stream=None):
        """Generated tokens [B, n] int32; negative entries are skipped."""
        self._add(1, tokens, None, slots, stream)

    def set_bias(self, tokens, values, slots=None, stream=None):
        """Biases values [B, n] fp32 of tokens [B, n] int32 (each token once)."""
        self._add(2, tokens, values, slots, stream)

    def accept(self, tokens, path, bonus, slots=None, stream=None):
        """Adds what a verification accepted: draft tokens [B, N+1], and its path [B, N]
        and bonus [B]."""
        import torch
        B, R = tokens.shape
        _check_in(tokens, torch.int32, (B, R), self.device, "tokens")
        _check_in(path, torch.int32, (B, R - 1), self.device, "path")
        _check_in(bonus, torch.int32, (B,), self.device, "bonus")
        self._call("tv_context_accept", B, R - 1, self._slots(slots, B), _at(tokens),
                   _at(path), _at(bonus), self.verifier._stream(stream))


class KVCache:
    """A paged key/value cache in 4 bits (tv_cache) and the attention over it: ``data``
    [layers, pages, kv_heads, 2, page_size * head_dim * 9 / 16] uint8 (keys, then values) and
    ``exponents`` [layers, 2, kv_heads] int32, zeros where none are given.  A request's
    tokens are found by ``lengths`` [B] int32 (tokens cached) and ``table`` [B, max_pages]
    int32 (its pages, in order).  Calls run on the given (default: current) stream."""

    def __init__(self, verifier, layers, pages, kv_heads, head_dim, page_size=64, data=None,
                 exponents=None):
        import torch
        if head_dim not in (64, 128):
            raise ValueError(f"head_dim: expected 64 or 128, got {head_dim}")
        if page_size not in (16, 32, 64, 128):
            raise ValueError(f"page_size: expected 16, 32, 64 or 128, got {page_size}")
        if min(layers, pages, kv_heads) < 1:
            raise ValueError("layers, pages and kv_heads: expected at least one of each")
        self.torch = torch                       # (an import statement a call costs 0.3 us each)
        self.verifier, self.device = verifier, verifier.device
        self.layers, self.pages, self.kv_heads = layers, pages, kv_heads
        self.head_dim, self.page_size = head_dim, page_size
        shape = (layers, pages, kv_heads, 2, page_size * head_dim * 9 // 16)
        dev = self.device
        self.data = torch.zeros(shape, dtype=torch.uint8, device=dev) if data is None else data
        self.exponents = torch.zeros(layers, 2, kv_heads, dtype=torch.int32, device=dev) \
            if exponents is None else exponents
        _check_in(self.data, torch.uint8, shape, dev, "data")
        _check_in(self.exponents, torch.int32, (layers, 2, kv_heads), dev, "exponents")
        self.struct = _Cache(layers, pages, kv_heads, head_dim, page_size, self.data.data_ptr(),
                             self.exponents.data_ptr())
        self.ref = ctypes.cast(ctypes.pointer(self.struct), _P)

    def _call(self, name, *args):
        rc = getattr(self.verifier.lib, name)(self.verifier.handle, self.ref, *args)
        if rc != 0:
            raise LibraryError(name, rc, self.verifier.lib)

    def _table(self, lengths, table, B):
        """The number of pages in a row of a page table that is one."""
        n = table.shape[1] if table.dim() == 2 else -1
        _check_in(lengths, self.torch.int32, (B,), self.device, "lengths")
        _check_in(table, self.torch.int32, (B, n), self.device, "table")
        return n

    def _kind(self, dtype):
        if dtype in ("bf16", self.torch.bfloat16):
            return TV_BF16, self.torch.bfloat16
        if dtype in ("fp32", self.torch.float32):
            return TV_FP32, self.torch.float32
        raise ValueError(f"dtype: expected bf16 or fp32, got {dtype}")

    def write(self, layer, k, v, lengths, table, rows=None, stream=None):
        """Quantises keys and values [B, R, kv_heads, head_dim] (bf16 or fp32) into the
        positions behind what is cached, row i of request b at lengths[b] + i; ``rows`` [B]
        int32 gives the rows of each request (default: all R).  Lengths do not change
        (tv_cache_write)."""
        B, R = k.shape[:2]
        code = self.verifier._float_code(k, "k")
        shape = (B, R, self.kv_heads, self.head_dim)
        _check_in(k, k.dtype, shape, self.device, "k")
        _check_in(v, k.dtype, shape, self.device, "v")
        n = self._table(lengths, table, B)
        if rows is not None:
            _check_in(rows, self.torch.int32, (B,), self.device, "rows")
        self._call("tv_cache_write", layer, B, R, code, k.data_ptr(), v.data_ptr(),
                   lengths.data_ptr(), table.data_ptr(), n, _at(rows),
                   self.verifier._stream(stream))

    def read(self, layer, lengths, table, n, first=None, dtype="bf16", out=None, stream=None):
        """Keys and values [B, n, kv_heads, head_dim] of positions first[b] + i < lengths[b]
        (``first`` [B] int32, default 0), zeros behind the last (tv_cache_read).  ``out`` =
        (k, v) to write into."""
        B = lengths.shape[0]
        pages = self._table(lengths, table, B)
        code, kind = self._kind(dtype)
        if first is not None:
            _check_in(first, self.torch.int32, (B,), self.device, "first")
        shape = (B, n, self.kv_heads, self.head_dim)
        k, v = self.verifier._empty(stream, (shape, kind), (shape, kind)) if out is None else out
        if out is not None:
            _check_out(k, kind, shape, self.device)
            _check_out(v, kind, shape, self.device)
        self._call("tv_cache_read", layer, B, n, code, lengths.data_ptr(), table.data_ptr(),
                   pages, _at(first), k.data_ptr(), v.data_ptr(),
                   self.verifier._stream(stream))
        return k, v

    def attend(self, layer, q, lengths, table, parents=None, rows=None, scale=None, out=None,
               stream=None):
        """Attention [B, R, heads, head_dim] bf16 of queries q of that shape over the cache:
        row i of request b, at position lengths[b] + i, sees what is cached, its ancestors in
        the tree ``parents`` [B, R] int32 (None: rows 0 to i) and itself; ``rows`` [B] int32
        gives the rows of each request (the output's others are 0), ``scale`` the factor of the
        scores (default head_dim ** -0.5).  heads is a multiple of kv_heads, whose query heads
        lie together (tv_tree_attention)."""
        B, R, heads = q.shape[:3]
        shape = (B, R, heads, self.head_dim)
        _check_in(q, self.torch.bfloat16, shape, self.device, "q")
        n = self._table(lengths, table, B)
        if parents is not None:
            _check_in(parents, self.torch.int32, (B, R), self.device, "parents")
        if rows is not None:
            _check_in(rows, self.torch.int32, (B,), self.device, "rows")
        if out is None:
            out, = self.verifier._empty(stream, (shape, self.torch.bfloat16))
        else:
            _check_out(out, self.torch.bfloat16, shape, self.device)
        self._call("tv_tree_attention", layer, B, R, heads, q.data_ptr(), lengths.data_ptr(),
                   table.data_ptr(), n, _at(parents), _at(rows),
                   float(scale) if scale is not None else self.head_dim ** -0.5,
                   out.data_ptr(), self.verifier._stream(stream))
        return out

    def accept(self, path, tau, lengths, table, out=None, stream=None):
        """After a verification with the paths [B, N] and tau [B] that it returned: moves, in
        every layer, the accepted nodes' rows behind the root's and returns the new lengths
        lengths + 1 + tau (tv_cache_accept); a tree marked invalid keeps its length.
        ``out`` [B] int32 to write them into, not ``lengths`` itself."""
        B, N = path.shape
        _check_in(path, self.torch.int32, (B, N), self.device, "path")
        _check_in(tau, self.torch.int32, (B,), self.device, "tau")
        n = self._table(lengths, table, B)
        if out is None:
            out, = self.verifier._empty(stream, ((B,), self.torch.int32))
        else:
            _check_out(out, self.torch.int32, (B,), self.device)
        self._call("tv_cache_accept", B, N, lengths.data_ptr(), table.data_ptr(), n,
                   path.data_ptr(), tau.data_ptr(), out.data_ptr(),
                   self.verifier._stream(stream))
        return out
