"""The training operators' row kernels, built for the host from their CUDA sources."""
from __future__ import annotations

import ctypes as C
import os
import shutil
import subprocess

import torch

from .translate import translate

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(os.path.dirname(HERE))
CSRC = os.path.join(ROOT, "paper_2609_36074_b200", "csrc")
HEADER = os.path.join(ROOT, "include", "gem_nlr.h")
TYPES = {"f32": (torch.float32, 0), "f16": (torch.float16, 1), "bf16": (torch.bfloat16, 2)}


def cuda_include():
    nvcc = shutil.which(os.environ.get("NVCC", "nvcc"))
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include") if nvcc else "/usr/local/cuda/include"
    return path if os.path.exists(os.path.join(path, "cuda_fp16.h")) else None


def build(folder, pairs):
    """{(file, type): library} of the translated kernels_<file>.cu for one element type each, compiled side by side."""
    started = []
    for name, kind in pairs:
        out = os.path.join(folder, f"{name}_{kind}")
        os.makedirs(out)
        translate(CSRC, HEADER, out, kind, polls=("400u", "50u"))
        lib = os.path.join(out, "kernels.so")
        started.append((name, kind, lib, subprocess.Popen(
            ["g++", "-std=c++17", "-O1", "-fPIC", "-shared", "-fpermissive", "-w", "-I" + cuda_include(), "-I" + out, "-I" + HERE,
             f'-DFILE_UNDER_TEST="kernels_{name}.cu"', os.path.join(out, "all.cpp"), "-o", lib],
            stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)))
    libs = {}
    for name, kind, lib, p in started:
        text, _ = p.communicate()
        if p.returncode:
            raise RuntimeError(text[-4000:])
        libs[name, kind] = Rows(lib, name, kind)
    return libs


class Rows:
    """One translated library: a region for each matrix that copies may read, the schedule's seed, then the C entry point."""

    def __init__(self, path, name, kind):
        L = self.L = C.CDLL(path)
        vp, i32, i64, f32, size = C.c_void_p, C.c_int32, C.c_int64, C.c_float, C.c_size_t
        self.dtype, self.type = TYPES[kind]
        L.emu_begin.argtypes = [i32, C.c_uint64, i32, i32]
        L.emu_region.argtypes = [vp, size]
        L.emu_report.restype = C.c_char_p
        if name == "norm":
            L.gem_nlr_layer_norm.argtypes = [vp, i32, i64, vp, vp, i32, i64, i32, f32, vp, i64, vp, vp, vp]
            L.gem_nlr_layer_norm_backward.argtypes = [vp, i64, vp, i64, i32, vp, vp, vp, i32, i64, i32, vp, i64, vp, vp, vp, size, vp]
            L.gem_nlr_layer_norm_backward_scratch_bytes.argtypes = [i64, i32]
            L.gem_nlr_layer_norm_backward_scratch_bytes.restype = size
        else:
            L.gem_nlr_label_cross_entropy.argtypes = [vp, i32, i64, vp, i64, i32, i32, vp, vp, vp, i64, vp, size, vp]
            L.gem_nlr_label_cross_entropy_scratch_bytes.argtypes = [i64, i32]
            L.gem_nlr_label_cross_entropy_scratch_bytes.restype = size

    def run(self, fn, *args, reads=(), resident=2, seed=1, lost=0, lost_message=0):
        """The return code; what the emulation recorded is in `report`."""
        self.L.emu_begin(resident, seed, lost, lost_message)
        for m in reads:
            if m is not None and m.numel():
                last = sum((n - 1) * s for n, s in zip(m.shape, m.stride()))
                self.L.emu_region(m.data_ptr(), (last + 1) * m.element_size())
        rc = getattr(self.L, "gem_nlr_" + fn)(*[a.data_ptr() if isinstance(a, torch.Tensor) else a for a in args], None)
        self.report = self.L.emu_report().decode()
        return rc

    def layer_norm(self, x, w, b, y, mean, rstd, eps=1e-5, **kw):
        return self.run("layer_norm", x, self.type, x.stride(0), w, b, 0 if w is None or w.dtype == torch.float32 else self.type, *x.shape,
                        eps, y, y.stride(0), mean, rstd, reads=(x,), **kw)

    def layer_norm_backward(self, dy, x, mean, rstd, w, dx, dw, db, **kw):
        size = self.L.gem_nlr_layer_norm_backward_scratch_bytes(*x.shape)
        scratch = flat(size, torch.uint8).fill_(0xff)
        return self.run("layer_norm_backward", dy, dy.stride(0), x, x.stride(0), self.type, mean, rstd, w,
                        0 if w is None or w.dtype == torch.float32 else self.type, *x.shape, dx, 0 if dx is None else dx.stride(0), dw, db,
                        scratch, size, reads=(dy, x, mean, rstd), **kw)

    def label_cross_entropy(self, z, labels, mean, loss, row, dz, **kw):
        size = self.L.gem_nlr_label_cross_entropy_scratch_bytes(*z.shape)
        scratch = flat(size, torch.uint8).fill_(0xff)
        return self.run("label_cross_entropy", z, self.type, z.stride(0), labels, *z.shape, int(mean), loss, row, dz,
                        0 if dz is None else dz.stride(0), scratch, size, reads=(z, labels), **kw)


def flat(numel, dtype):
    """numel elements that begin at a multiple of 256 bytes."""
    size = torch.empty(0, dtype=dtype).element_size()
    memory = torch.empty(numel * size + 256, dtype=torch.uint8)
    at = -memory.data_ptr() % 256
    return memory[at:at + numel * size].view(dtype)


class Matrix:
    """n x d with rows ld apart that begin `first` elements into memory full of `around`."""

    def __init__(self, n, d, dtype, ld, first, around):
        self.whole = flat(first + (n - 1) * ld + d + 16, dtype).fill_(around)
        self.m = self.whole.as_strided((n, d), (ld, 1), self.whole.storage_offset() + first)
        self.around = around
        outside = torch.ones(self.whole.numel(), dtype=torch.bool)
        outside.as_strided((n, d), (ld, 1), first).fill_(False)
        self.outside = outside

    def kept(self):
        """Whether nothing was written beside the matrix."""
        v = self.whole[self.outside]
        return bool((v.isnan() if self.around != self.around else v == self.around).all())
