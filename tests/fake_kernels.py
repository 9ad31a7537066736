"""FakeCuda that also names the kernels (fake_kernels.cpp)."""
import ctypes
import glob
import os
import subprocess

from conftest import ROOT
from fake_cuda import FakeCuda


class FakeKernels(FakeCuda):
    def __init__(self, folder):
        from paper_2608_26581_gb300 import _build, rfq
        _build.build()
        nvcc = os.path.realpath(_build._nvcc())
        path = os.path.join(str(folder), "librfq_fake_kernels.so")
        r = subprocess.run(["g++", "-O1", "-std=c++17", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-o", path, "-I",
                            os.path.join(os.path.dirname(os.path.dirname(nvcc)), "include"),
                            os.path.join(ROOT, "tests", "fake_kernels.cpp"), *sorted(glob.glob(os.path.join(_build.BUILD, "*.o")))],
                           capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-3000:]
        self.lib = ctypes.CDLL(path)
        for name in rfq.EXPORTED:            # the types that the binding gives them
            real = getattr(rfq.load_library(), name)
            f = getattr(self.lib, name)
            f.restype, f.argtypes = real.restype, real.argtypes
        for f in (self.lib.fake_kernel, self.lib.fake_launched_kernel):
            f.restype, f.argtypes = ctypes.c_char_p, [ctypes.c_int]

    def kernels(self):
        """The names of the library's kernels."""
        return [self.lib.fake_kernel(i).decode() for i in range(self.lib.fake_kernels())]

    def call(self, f, *args):
        """(status, [(kernel, grid x, y, z, threads, cluster, shared bytes)]) of one call."""
        n, k = self.lib.fake_launches(), self.lib.fake_launched()
        status = getattr(self.lib, f)(*args)
        shapes, more = self.launches()[n:], self.lib.fake_launched() - k
        assert more == len(shapes)
        return status, [(self.lib.fake_launched_kernel(k + i).decode(), *s) for i, s in enumerate(shapes)]
