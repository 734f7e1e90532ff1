"""ctypes marshalling for libfade.so (names mirror include/fade.h). Device buffers are torch tensors on the
context's device; host buffers are numpy arrays."""
import ctypes as C
import os
import struct

import numpy as np

from .buildlib import LIB

F32, BF16 = 0, 1
TOKEN_U8, TOKEN_I32, TOKEN_I64 = 0, 1, 2
NORMS = {"none": 0, "layer": 1, "rms": 2}
FROZEN, ONLINE_ADAM = 0, 1
ABI_VERSION = 2
TAPS = ["X", "CACHE", "H_GLOBAL", "H_LOCAL", "ALPHA", "H_MIX", "Y_DOWN", "Z_BMM", "H_A", "H_COARSE", "H_EXPAND",
        "H_OUT", "LOGITS", "PROBS"]


class Config(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("abi_version", C.c_uint32),
                ("B", C.c_uint32), ("T", C.c_uint32), ("D", C.c_uint32), ("H", C.c_uint32),
                ("d_low", C.c_uint32), ("cache_chunk", C.c_uint32), ("conv_k", C.c_uint32),
                ("d_cache", C.c_uint32), ("d_e", C.c_uint32), ("ablation", C.c_uint32),
                ("dtype", C.c_uint32), ("update_mode", C.c_uint32),
                ("lr", C.c_float), ("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float),
                ("device", C.c_int32), ("hip_stream", C.c_void_p)]


class JoinArgs(C.Structure):
    _fields_ = [("struct_size", C.c_uint32), ("norm_u", C.c_uint32), ("norm_n", C.c_uint32), ("eps", C.c_float),
                ("rows", C.c_size_t), ("width", C.c_size_t),
                ("stream_type", C.c_uint32), ("branch_type", C.c_uint32), ("lam_count", C.c_uint32), ("accumulate", C.c_uint32),
                ("lam", C.c_void_p), ("gamma_u", C.c_void_p), ("beta_u", C.c_void_p), ("gamma_n", C.c_void_p), ("beta_n", C.c_void_p),
                ("r", C.c_void_p), ("u", C.c_void_p), ("g", C.c_void_p),
                ("r_ld", C.c_size_t), ("u_ld", C.c_size_t), ("g_ld", C.c_size_t),
                ("h", C.c_void_p), ("n", C.c_void_p), ("h_ld", C.c_size_t), ("n_ld", C.c_size_t),
                ("keep_r", C.c_void_p), ("keep_u", C.c_void_p), ("keep_g", C.c_void_p), ("keep_n", C.c_void_p),
                ("dh", C.c_void_p), ("dn", C.c_void_p), ("dh_ld", C.c_size_t), ("dn_ld", C.c_size_t),
                ("dr", C.c_void_p), ("du", C.c_void_p), ("dg", C.c_void_p),
                ("dr_ld", C.c_size_t), ("du_ld", C.c_size_t), ("dg_ld", C.c_size_t),
                ("d_lam", C.c_void_p), ("d_gamma_u", C.c_void_p), ("d_beta_u", C.c_void_p), ("d_gamma_n", C.c_void_p), ("d_beta_n", C.c_void_p),
                ("work", C.c_void_p), ("work_bytes", C.c_size_t)]


def make_config(B, T, D, H, d_low=0, cache_chunk=0, conv_k=0, dtype=BF16, update_mode=FROZEN, lr=0.0, beta1=0.0,
                beta2=0.0, eps=0.0, device=0, hip_stream=None, d_cache=0, d_e=0, ablation=0):
    c = Config()
    c.struct_size = C.sizeof(Config)
    c.abi_version = ABI_VERSION
    c.B, c.T, c.D, c.H = B, T, D, H
    c.d_low, c.cache_chunk, c.conv_k = d_low, cache_chunk, conv_k
    c.d_cache, c.d_e, c.ablation = d_cache, d_e, ablation
    c.dtype, c.update_mode = dtype, update_mode
    c.lr, c.beta1, c.beta2, c.eps = lr, beta1, beta2, eps
    c.device, c.hip_stream = device, hip_stream
    return c


_lib = None


def lib():
    """Load libfade.so. Fails loudly when it has not been built (python -m paper_2604_07239_amd.buildlib)."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB):
            raise FadeError(-7, f"{LIB} is not built: run paper_2604_07239_amd.build() (hipcc, gfx950) first")
        L = C.CDLL(LIB)
        vp, sz = C.c_void_p, C.c_size_t
        L.fade_weights_nbytes.restype = sz
        L.fade_weights_nbytes.argtypes = [C.POINTER(Config)]
        L.fade_create.argtypes = [C.POINTER(Config), C.POINTER(vp)]
        L.fade_load_weights.argtypes = [vp, vp, sz]
        L.fade_reset.argtypes = [vp]
        L.fade_step_probs.argtypes = [vp, vp, vp, vp, vp]
        L.fade_step_update.argtypes = [vp, vp, vp]
        L.fade_encode_bound.restype = sz
        L.fade_encode_bound.argtypes = [vp, sz]
        L.fade_encode.argtypes = [vp, vp, sz, vp, sz, C.POINTER(sz)]
        L.fade_decode.argtypes = [vp, vp, sz, vp, sz, C.POINTER(sz)]
        L.fade_encode_device.argtypes = [vp, vp, sz, sz, sz]
        L.fade_payloads.argtypes = [vp, vp, vp, sz, C.POINTER(sz)]
        L.fade_decode_device.argtypes = [vp, vp, vp, sz, vp, sz, sz, sz]
        L.fade_quantize.argtypes = [vp, vp, sz, vp]
        L.fade_coder_encode_tables.argtypes = [vp, vp, vp, sz, sz, vp, sz, vp]
        L.fade_coder_decode_tables.argtypes = [vp, vp, sz, sz, vp, sz, vp, vp]
        L.fade_coder_encode_tables_noalloc.argtypes = [vp, vp, vp, sz, sz, vp, sz, vp]
        i, f = C.c_int, C.c_float
        L.fade_embed.argtypes = [vp, vp, i, sz, vp, i, sz, sz, sz, f, vp, i, sz]
        L.fade_embed_grad_work.restype = sz
        L.fade_embed_grad_work.argtypes = [sz, sz, sz]
        L.fade_embed_grad.argtypes = [vp, vp, i, sz, vp, i, sz, f, vp, sz, sz, sz, i, vp, sz]
        L.fade_checkpoint_nbytes.restype = sz
        L.fade_checkpoint_nbytes.argtypes = [sz, sz]
        L.fade_checkpoint.argtypes = [vp, vp, i, sz, sz, sz, vp]
        L.fade_checkpoint_read.argtypes = [vp, vp, sz, sz, vp, i, sz]
        L.fade_checkpoint_weight_grad_work.restype = sz
        L.fade_checkpoint_weight_grad_work.argtypes = [sz, sz, sz]
        L.fade_checkpoint_weight_grad.argtypes = [vp, vp, sz, sz, vp, i, sz, sz, vp, sz, i, vp, sz]
        L.fade_join_grad_work.restype = sz
        L.fade_join_grad_work.argtypes = [sz, sz]
        L.fade_join.argtypes = [vp, vp]
        L.fade_join_grad.argtypes = [vp, vp]
        L.fade_tap.restype = sz
        L.fade_tap.argtypes = [vp, C.c_int, vp, sz]
        L.fade_get_weights.argtypes = [vp, vp, sz]
        L.fade_debug_grad.argtypes = [vp, vp, sz]
        L.fade_profile.argtypes = [vp, C.c_int]
        L.fade_profile_read.argtypes = [vp, C.POINTER(C.c_char_p), C.POINTER(C.c_double), C.POINTER(C.c_uint64), C.c_int]
        L.fade_last_error.restype = C.c_char_p
        L.fade_last_error.argtypes = [vp]
        L.fade_destroy.argtypes = [vp]
        _lib = L
    return _lib


class FadeError(RuntimeError):
    def __init__(self, code, msg=""):
        super().__init__(f"libfade error {code}: {msg}")
        self.code = code


def weights_nbytes(cfg):
    return lib().fade_weights_nbytes(C.byref(cfg))


def _hp(a):
    return None if a is None else a.ctypes.data_as(C.c_void_p)


def _dp(t):
    return None if t is None else C.c_void_p(t.data_ptr())


# fade_join_args, packed in one go: a call from Python costs what its argument handling costs (fields one by one: 14 us a call)
_JOIN = struct.Struct("@3If2Q4I5P3P3Q2P2Q4P2P2Q3P3Q5PPQ")
assert _JOIN.size == C.sizeof(JoinArgs)
_NO_GRADS = (0,) * 17
_TYPES, _TOKENS = {}, {}


def _late_type(table, t):
    """torch is the caller's: its types are looked up when the first tensor comes."""
    if not _TYPES:
        import torch
        _TOKENS.update({torch.uint8: TOKEN_U8, torch.int32: TOKEN_I32, torch.int64: TOKEN_I64})
        _TYPES.update({torch.float32: F32, torch.bfloat16: BF16})  # last: another thread takes it for both
    return table.get(t.dtype)


class Fade:
    """One libfade context (see include/fade.h for the meaning of every call)."""

    def __init__(self, cfg):
        self.cfg = cfg
        self.L = lib()
        h = C.c_void_p()
        rc = self.L.fade_create(C.byref(cfg), C.byref(h))
        if rc:
            raise FadeError(rc, "fade_create")
        self.h = h
        self.B, self.T, self.device = cfg.B, cfg.T, cfg.device

    def _chk(self, rc):
        if rc:
            raise FadeError(rc, self.L.fade_last_error(self.h).decode())

    def close(self):
        if getattr(self, "h", None):
            self.L.fade_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- weights / state -------------------------------------------------------------------------
    def load_weights(self, blob):
        blob = np.ascontiguousarray(blob, dtype=np.float32)
        self._chk(self.L.fade_load_weights(self.h, _hp(blob), blob.nbytes))

    def reset(self):
        self._chk(self.L.fade_reset(self.h))

    def get_weights(self):
        n = weights_nbytes(self.cfg)
        out = np.zeros(n // 4, np.float32)
        self._chk(self.L.fade_get_weights(self.h, _hp(out), n))
        return out

    def debug_grad(self):
        n = weights_nbytes(self.cfg)
        out = np.zeros(n // 4, np.float32)
        self._chk(self.L.fade_debug_grad(self.h, _hp(out), n))
        return out

    # -- the step --------------------------------------------------------------------------------
    def step_probs(self, windows_dev, active_dev=None, freq_dev=None, probs_dev=None):
        self._chk(self.L.fade_step_probs(self.h, _dp(windows_dev), _dp(active_dev), _dp(freq_dev), _dp(probs_dev)))

    def step_update(self, targets_dev, active_dev=None):
        self._chk(self.L.fade_step_update(self.h, _dp(targets_dev), _dp(active_dev)))

    def tap(self, name):
        which = TAPS.index(name)
        width = self.L.fade_tap(self.h, which, None, 0)
        if width == 0:
            return None
        out = np.zeros((self.B, width), np.float32)
        if self.L.fade_tap(self.h, which, _hp(out), out.size) != width:
            raise FadeError(-7, "fade_tap")
        return out

    # -- compress / decompress -------------------------------------------------------------------
    def encode_bound(self, n):
        return self.L.fade_encode_bound(self.h, n)

    def encode(self, src):
        src = np.ascontiguousarray(src, dtype=np.uint8)
        cap = self.encode_bound(src.size)
        dst = np.zeros(cap, np.uint8)
        n = C.c_size_t()
        self._chk(self.L.fade_encode(self.h, _hp(src), src.size, _hp(dst), cap, C.byref(n)))
        return dst[:n.value].copy()

    def decode(self, blob, cap):
        blob = np.ascontiguousarray(blob, dtype=np.uint8)
        dst = np.zeros(max(cap, 1), np.uint8)
        n = C.c_size_t()
        self._chk(self.L.fade_decode(self.h, _hp(blob), blob.size, _hp(dst), cap, C.byref(n)))
        return dst[:n.value].copy()

    def encode_device(self, src_dev, n, first_step=0, n_steps=0):
        self._chk(self.L.fade_encode_device(self.h, _dp(src_dev), n, first_step, n_steps))

    def payloads(self):
        lens = np.zeros(self.B, np.uint32)
        total = C.c_size_t()
        rc = self.L.fade_payloads(self.h, _hp(lens), None, 0, C.byref(total))
        if rc not in (0, -5):
            self._chk(rc)
        data = np.zeros(max(total.value, 1), np.uint8)
        self._chk(self.L.fade_payloads(self.h, _hp(lens), _hp(data), data.size, C.byref(total)))
        return lens, data[:total.value]

    def decode_device(self, lens, data, dst_dev, n, first_step=0, n_steps=0):
        if first_step == 0:
            lens = np.ascontiguousarray(lens, dtype=np.uint32)
            data = np.ascontiguousarray(data, dtype=np.uint8)
            self._chk(self.L.fade_decode_device(self.h, _hp(lens), _hp(data) if data.size else None, data.size,
                                                _dp(dst_dev), n, 0, n_steps))
        else:
            self._chk(self.L.fade_decode_device(self.h, None, None, 0, _dp(dst_dev), n, first_step, n_steps))

    # -- stand-alone integer kernels -------------------------------------------------------------
    def quantize(self, probs_dev, freq_dev):
        rows = probs_dev.numel() // 256
        self._chk(self.L.fade_quantize(self.h, _dp(probs_dev), rows, _dp(freq_dev)))

    def coder_encode_tables(self, freq_dev, sym_dev, n_steps, n_streams, out_dev, cap, len_dev):
        self._chk(self.L.fade_coder_encode_tables(self.h, _dp(freq_dev), _dp(sym_dev), n_steps, n_streams, _dp(out_dev), cap, _dp(len_dev)))

    def coder_encode_tables_noalloc(self, freq_dev, sym_dev, n_steps, n_streams, out_dev, cap, len_dev):
        self._chk(self.L.fade_coder_encode_tables_noalloc(self.h, _dp(freq_dev), _dp(sym_dev), n_steps, n_streams, _dp(out_dev), cap, _dp(len_dev)))

    def coder_decode_tables(self, freq_dev, n_steps, n_streams, in_dev, cap, len_dev, sym_dev):
        self._chk(self.L.fade_coder_decode_tables(self.h, _dp(freq_dev), n_steps, n_streams, _dp(in_dev), cap, _dp(len_dev), _dp(sym_dev)))

    # -- operators around a program's own model -----------------------------------------------------
    # Tensors are checked here for what the C ABI cannot see: their device, type, shape and strides. Everything is enqueued on
    # the context's stream; nothing is allocated. On which of torch's streams a tensor was written is not looked at: give make_config the stream of the
    # program's other work (hip_stream=stream.cuda_stream; 1 for torch's default stream, whose handle of 0 stands for none), or order the two by events. A
    # context's own stream (hip_stream=None) and torch's default one wait for each other, at some 20 us a change.
    def _bad(self, what):
        raise FadeError(-1, what)

    def _rows(self, t, name, rows=None, width=None):
        """(pointer, type, ld) of a matrix [rows][width] whose columns are neighbours."""
        kind = _TYPES.get(t.dtype)
        if kind is None:
            kind = _late_type(_TYPES, t)
        if kind is None or t.dim() != 2 or t.get_device() != self.device:
            self._bad(f"{name}: a matrix of float32 or bfloat16 on the context's device is needed")
        n, w = t.shape
        if (rows is not None and n != rows) or (width is not None and w != width):
            self._bad(f"{name}: shape {(n, w)} where [{rows}, {width}] is needed")
        ld, step = t.stride()
        if step != 1 and w > 1:
            self._bad(f"{name}: neighbouring columns have to be neighbours in memory")
        return t.data_ptr(), kind, ld if n > 1 else w

    def _same(self, t, name, rows, width, kind):
        """(pointer, ld) of a matrix of a known type, or of none."""
        if t is None:
            return 0, 0
        p, k, ld = self._rows(t, name, rows, width)
        if k != kind:
            self._bad(f"{name}: another type than the other matrices of its side")
        return p, ld

    def _vector(self, t, name, count):
        if t is None:
            return 0
        kind = _TYPES.get(t.dtype)
        if kind is None:
            kind = _late_type(_TYPES, t)
        if kind != F32 or t.get_device() != self.device or t.numel() != count or not t.is_contiguous():
            self._bad(f"{name}: {count} contiguous float32 values on the context's device are needed")
        return t.data_ptr()

    def _bytes(self, t, name, least):
        """(pointer, size) of a buffer of at least `least` bytes."""
        size = t.nbytes
        if t.get_device() != self.device or not t.is_contiguous() or size < least:
            self._bad(f"{name}: a contiguous buffer of {least} bytes on the context's device is needed")
        return t.data_ptr(), size

    def _tokens(self, t):
        kind = _TOKENS.get(t.dtype)
        if kind is None:
            kind = _late_type(_TOKENS, t)
        if kind is None or t.get_device() != self.device or not t.is_contiguous():
            self._bad("tokens: contiguous uint8, int32 or int64 values on the context's device are needed")
        return t.data_ptr(), kind, t.numel()

    def _grad(self, t, width=None):
        """(pointer, ld) of a gradient: a matrix of float32."""
        p, kind, ld = self._rows(t, "grad", None, width)
        if kind != F32:
            self._bad("grad: float32 is needed")
        return p, ld

    def embed(self, tokens, table, out, scale=1.0):
        """out[i] = scale * table[tokens[i]]; tokens outside the table give zeros."""
        tp, tk, n = self._tokens(tokens)
        ep, ek, eld = self._rows(table, "table")
        op, ok, old = self._rows(out, "out", n, table.shape[1])
        self._chk(self.L.fade_embed(self.h, tp, tk, n, ep, ek, eld, table.shape[0], table.shape[1], scale, op, ok, old))

    def embed_grad_work(self, n, vocab, width):
        return self.L.fade_embed_grad_work(n, vocab, width)

    def embed_grad(self, tokens, dout, grad, work, scale=1.0, accumulate=False):
        """grad[v] = scale * sum of dout[i] where tokens[i] == v, or that added to grad."""
        tp, tk, n = self._tokens(tokens)
        gp, gld = self._grad(grad)
        vocab, width = grad.shape
        dp, dk, dld = self._rows(dout, "dout", n, width)
        wp, wn = self._bytes(work, "work", 0)
        self._chk(self.L.fade_embed_grad(self.h, tp, tk, n, dp, dk, dld, scale, gp, gld, vocab, width, int(accumulate), wp, wn))

    def checkpoint_nbytes(self, rows, width):
        return self.L.fade_checkpoint_nbytes(rows, width)

    def checkpoint(self, x, keep):
        """Writes the 8-bit checkpoint of x [rows][width] into keep (checkpoint_nbytes(rows, width) bytes)."""
        xp, xk, xld = self._rows(x, "x")
        rows, width = x.shape
        self._chk(self.L.fade_checkpoint(self.h, xp, xk, xld, rows, width, self._bytes(keep, "keep", self.L.fade_checkpoint_nbytes(rows, width))[0]))

    def checkpoint_read(self, keep, out):
        """The values a checkpoint stands for into out [rows][width]."""
        op, ok, old = self._rows(out, "out")
        rows, width = out.shape
        kp, _ = self._bytes(keep, "keep", self.L.fade_checkpoint_nbytes(rows, width))
        self._chk(self.L.fade_checkpoint_read(self.h, kp, rows, width, op, ok, old))

    def checkpoint_weight_grad_work(self, rows, in_width, out_width):
        return self.L.fade_checkpoint_weight_grad_work(rows, in_width, out_width)

    def checkpoint_weight_grad(self, keep, dy, grad, work, accumulate=False):
        """grad [in][out] = x^T dy from the checkpoint of x [rows][in] and dy [rows][out], or that added to grad."""
        dp, dk, dld = self._rows(dy, "dy")
        rows, n = dy.shape
        gp, gld = self._grad(grad, n)
        k = grad.shape[0]
        kp, _ = self._bytes(keep, "keep", self.L.fade_checkpoint_nbytes(rows, k))
        wp, wn = self._bytes(work, "work", 0)
        self._chk(self.L.fade_checkpoint_weight_grad(self.h, kp, rows, k, dp, dk, dld, n, gp, gld, int(accumulate), wp, wn))

    def _join_model(self, width, norm_u, norm_n, eps, lam, gamma_u, beta_u, gamma_n, beta_n):
        if norm_u not in NORMS or norm_n not in NORMS:
            self._bad(f"norm: one of {', '.join(NORMS)} is needed")
        if not abs(eps) <= 3.4028234663852886e38:  # what is past fp32 can't be packed; the rest is the library's to refuse
            self._bad("eps: a number of fp32 is needed")
        count = 0
        if lam is not None:
            count = lam.numel()
            if count != 1 and count != width:
                self._bad(f"lam: 1 or {width} values are needed")
        v = self._vector
        return count, (v(lam, "lam", count), v(gamma_u, "gamma_u", width), v(beta_u, "beta_u", width), v(gamma_n, "gamma_n", width), v(beta_n, "beta_n", width))

    def _keep(self, t, rows, width):
        return 0 if t is None else self._bytes(t, "keep", self.L.fade_checkpoint_nbytes(rows, width))[0]

    def join(self, h, n=None, *, r, u, g=None, lam=None, norm_u="layer", norm_n="layer", gamma_u=None, beta_u=None, gamma_n=None, beta_n=None, eps=0.0,
             keep_r=None, keep_u=None, keep_g=None, keep_n=None):
        """h = lam * r + sigma(g) * norm_u(u) and n = norm_n(h), and 8-bit checkpoints of r, u, g and n where buffers are given."""
        rp, stream, rl = self._rows(r, "r")
        rows, width = r.shape
        hp, hl = self._same(h, "h", rows, width, stream)
        up, branch, ul = self._rows(u, "u", rows, width)
        gp, gl = self._same(g, "g", rows, width, branch)
        np_, nl = self._same(n, "n", rows, width, branch)
        count, params = self._join_model(width, norm_u, norm_n, eps, lam, gamma_u, beta_u, gamma_n, beta_n)
        k = self._keep
        a = _JOIN.pack(_JOIN.size, NORMS[norm_u], NORMS[norm_n], eps, rows, width, stream, branch, count, 0, *params, rp, up, gp, rl, ul, gl, hp, np_, hl, nl,
                       k(keep_r, rows, width), k(keep_u, rows, width), k(keep_g, rows, width), k(keep_n, rows, width), *_NO_GRADS)
        self._chk(self.L.fade_join(self.h, a))

    def join_grad_work(self, rows, width):
        return self.L.fade_join_grad_work(rows, width)

    def join_grad(self, dh, dn, work, *, r=None, u=None, g=None, keep_r=None, keep_u=None, keep_g=None, lam=None, norm_u="layer", norm_n="layer", gamma_u=None,
                  beta_u=None, gamma_n=None, beta_n=None, eps=0.0, dr=None, du=None, dg=None, d_lam=None, d_gamma_u=None, d_beta_u=None, d_gamma_n=None,
                  d_beta_n=None, accumulate=False):
        """The gradients of join() for those of h and n (either may be None), from its operands or from their checkpoints. The block had a gate if g or keep_g
        is given: without them these are the gradients of a block that had none."""
        like = dh if dh is not None else dn
        if like is None:
            self._bad("neither dh nor dn")
        if like.dim() != 2:
            self._bad("dh or dn: a matrix is needed")
        rows, width = like.shape
        # the type of each side is that of the first matrix given; a side that nobody gives has any type that goes with the other's
        first_s = r if r is not None else dh if dh is not None else dr
        first_b = u if u is not None else dn if dn is not None else du if du is not None else g if g is not None else dg
        branch = self._rows(first_b, "the branch's matrices", rows, width)[1] if first_b is not None else None
        stream = self._rows(first_s, "the stream's matrices", rows, width)[1] if first_s is not None else branch
        if branch is None:
            branch = stream
        m = self._same
        (rp, rl), (dhp, dhl), (drp, drl) = m(r, "r", rows, width, stream), m(dh, "dh", rows, width, stream), m(dr, "dr", rows, width, stream)
        (up, ul), (gp, gl), (dnp, dnl) = m(u, "u", rows, width, branch), m(g, "g", rows, width, branch), m(dn, "dn", rows, width, branch)
        (dup, dul), (dgp, dgl) = m(du, "du", rows, width, branch), m(dg, "dg", rows, width, branch)
        count, params = self._join_model(width, norm_u, norm_n, eps, lam, gamma_u, beta_u, gamma_n, beta_n)
        v, k = self._vector, self._keep
        a = _JOIN.pack(_JOIN.size, NORMS[norm_u], NORMS[norm_n], eps, rows, width, stream, branch, count, int(accumulate), *params, rp, up, gp, rl, ul, gl, 0, 0, 0, 0,
                       k(keep_r, rows, width), k(keep_u, rows, width), k(keep_g, rows, width), 0, dhp, dnp, dhl, dnl, drp, dup, dgp, drl, dul, dgl,
                       v(d_lam, "d_lam", count), v(d_gamma_u, "d_gamma_u", width), v(d_beta_u, "d_beta_u", width), v(d_gamma_n, "d_gamma_n", width),
                       v(d_beta_n, "d_beta_n", width), *self._bytes(work, "work", 0))
        self._chk(self.L.fade_join_grad(self.h, a))

    # -- profiling -------------------------------------------------------------------------------
    def profile(self, enable):
        self._chk(self.L.fade_profile(self.h, 1 if enable else 0))

    def profile_read(self):
        cap = 64
        names = (C.c_char_p * cap)()
        ms = (C.c_double * cap)()
        cnt = (C.c_uint64 * cap)()
        n = self.L.fade_profile_read(self.h, names, ms, cnt, cap)
        return {names[i].decode(): (ms[i], cnt[i]) for i in range(n)}
