"""Loader for the CPU build of the training operators (tests/emu/train_emu.cpp) and tensors in guarded buffers.  Test scaffolding only."""
import ctypes as C
import os
import subprocess

import torch

from paper_1911_11377_amd import build as lib_build
from paper_1911_11377_amd import ckksmi

HERE = os.path.dirname(os.path.abspath(__file__))
EMU = os.path.join(HERE, "emu")
LIB = os.path.join(EMU, "libckksmi_train_emu.so")
CLANG = os.path.join(os.path.dirname(lib_build.HIPCC), "..", "llvm", "bin", "clang++")  # a host compiler with both 16-bit types

available = os.path.exists(CLANG)


def build():
    src = os.path.join(EMU, "train_emu.cpp")
    deps = [src] + [os.path.join(EMU, f) for f in ("hip_emu.h", "train_emu.h")] + [os.path.join(lib_build.CSRC, f) for f in os.listdir(lib_build.CSRC)]
    deps += [os.path.join(HERE, "..", "include", f) for f in ("ckksmi.h", "ckksmi_train.h", "ckksmi_profile.h")]
    if os.path.exists(LIB) and all(os.path.getmtime(LIB) >= os.path.getmtime(d) for d in deps):
        return LIB
    tmp = LIB + ".tmp.%d" % os.getpid()
    subprocess.check_call([CLANG, "-O1", "-g", "-std=c++17", "-fPIC", "-shared", "-ffp-contract=off", "-DCKKSMI_EMULATE", "-include", os.path.join(EMU, "train_emu.h"),
                           "-Wno-unknown-attributes", "-Wno-pass-failed", "-x", "c++", src, "-o", tmp])
    os.replace(tmp, LIB)
    return LIB


class EmuContext:
    """what the plans of training.py use of a context"""

    def __init__(self):
        path = build()
        self._L = C.CDLL(path)
        for name, args in ckksmi.SIGNATURES.items():
            if name.startswith(ckksmi.TRAINING):
                getattr(self._L, name).argtypes = args
        self._L.emu_train_context.restype = C.c_void_p
        self._L.emu_train_context_free.argtypes = [C.c_void_p]
        self._L.emu_alloc.restype = C.c_void_p
        self._L.emu_alloc.argtypes = [C.c_size_t]
        self._L.emu_free.argtypes = [C.c_void_p]
        self._L.emu_errors.restype = C.c_long
        self._h = self._L.emu_train_context()

    def errors(self):
        return self._L.emu_errors()

    def close(self):
        self._L.emu_train_context_free(self._h)

    def _call(self, name, *args):
        rc = getattr(self._L, name)(*args)
        if rc != ckksmi.OK:
            raise ckksmi.CkksmiError(rc, name)
        return rc

    @staticmethod
    def _stream(stream):
        return None

    def guarded(self, t):
        """a copy of t whose end (to 16 bytes) lies against a page that cannot be touched"""
        n = t.numel() * t.element_size()
        addr = self._L.emu_alloc(max(n, 1))
        raw = (C.c_uint8 * max(n, 1)).from_address(addr)
        out = torch.frombuffer(raw, dtype=torch.uint8)[:n].view(t.dtype).view(t.shape) if n else t.clone()
        out.copy_(t)
        return out
