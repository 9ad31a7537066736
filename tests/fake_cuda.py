"""The library linked against fake_cuda_runtime.cpp: its entry points with
nothing behind them but the host code."""
import ctypes
import glob
import os
import subprocess

from conftest import ROOT


class FakeCuda:
    def __init__(self, folder):
        from paper_2608_26581_gb300 import _build, rfq
        _build.build()
        nvcc = os.path.realpath(_build._nvcc())
        path = os.path.join(str(folder), "librfq_fake.so")
        r = subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-o", path, "-I",
                            os.path.join(os.path.dirname(os.path.dirname(nvcc)), "include"),
                            os.path.join(ROOT, "tests", "fake_cuda_runtime.cpp"), *sorted(glob.glob(os.path.join(_build.BUILD, "*.o")))],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        self.lib = ctypes.CDLL(path)
        for name in rfq.EXPORTED:            # the types that the binding gives them
            real = getattr(rfq.load_library(), name)
            f = getattr(self.lib, name)
            f.restype, f.argtypes = real.restype, real.argtypes

    def device(self, d):
        self.lib.fake_device(d)

    def launches(self):
        """(grid x, y, z, threads, cluster, shared bytes) of each launch so far"""
        out = []
        for i in range(self.lib.fake_launches()):
            v = (ctypes.c_uint * 6)()
            self.lib.fake_launch(i, v)
            out.append(tuple(v))
        return out
