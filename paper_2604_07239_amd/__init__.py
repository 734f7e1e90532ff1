"""FADE's batched probability step and arithmetic coder on one MI355X: thin ctypes binding of libfade.so.

Every function here only marshals arguments; all arithmetic of the path runs in the HIP kernels behind the
C ABI declared in include/fade.h. There is no CPU fallback: without the built library or without a GPU the
calls raise.
"""
from .binding import (BF16, F32, FROZEN, NORMS, ONLINE_ADAM, TAPS, TOKEN_I32, TOKEN_I64, TOKEN_U8, Config, Fade,  # noqa: F401
                      FadeError, JoinArgs, lib, make_config, weights_nbytes)
from .buildlib import LIB, build  # noqa: F401

ONLINE_SUPPORTED = True
