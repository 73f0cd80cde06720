"""The double-precision exponential that sums for a border are made with, against the host's extended precision.

Bound, relative to the value: the reduced argument is off by the roundings of two fused operations on numbers of at most
ln 2 / 2 < 0.35, 2^-55 each, together 2^-54 of the value.  The last step of the polynomial rounds a number from 0.707 to
1.42 to half of a step, 2^-53 (2^-54 below 1); the one in front of it a number below 1.21, which r = 0.35 at most multiplies;
each earlier one weighs a third of the next or less.  Above 1 that is 2^-53 (1 + 0.35 + 0.07) and 2^-54, below 1 2^-54 (1 + 0.35 + 0.07) / 0.707 and
2^-54: less than 2^-52 in both cases.  The series' rest is below 5e-18 / 0.707."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest
import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

pytestmark = pytest.mark.gpu

_SOURCE = r"""
#include "fsd_truncate.cuh"
namespace {
__global__ void exp_kernel(const double* x, double* y, int n) {
    const int i = blockIdx.x * blockDim.x + threadIdx.x;
    if (i < n) y[i] = fsd::exp_of(x[i]);
}
}
extern "C" int run(const double* x, double* y, int n) {
    exp_kernel<<<(n + 255) / 256, 256>>>(x, y, n);
    return cudaDeviceSynchronize() == cudaSuccess ? 0 : 1;
}
"""


def test_the_exponential_of_the_sums(tmp_path):
    from paper_2502_20704_b200 import build
    (tmp_path / "exp.cu").write_text(_SOURCE)
    lib = str(tmp_path / "exp.so")
    nvcc = os.environ.get("NVCC", "nvcc")
    assert shutil.which(nvcc), "nvcc is needed"
    subprocess.run([nvcc, *build.NVCC_FLAGS, "-I", os.path.join(ROOT, "include"), "-I", build.CSRC, "-o", lib, str(tmp_path / "exp.cu")], check=True)
    rng = np.random.default_rng(1)
    x = np.concatenate([-rng.random(400000) * 700, -rng.random(200000), -np.exp(-rng.random(100000) * 40), rng.random(50000) * 700,
                        -np.arange(2000) * np.log(2) / 2, -np.arange(2000) * np.log(2) / 2 * (1 + 2.0 ** -40), [-700.0, 0.0, -0.0, 700.0]])
    x = x[x >= -700]
    rest = np.array([-np.inf, -1e300, np.nextafter(-700.0, -701), np.nan])
    dx = torch.from_numpy(np.concatenate([x, rest])).cuda()
    dy = torch.full_like(dx, 7.0)
    f = ctypes.CDLL(lib).run
    f.argtypes = [ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int]
    torch.cuda.synchronize()
    assert f(dx.data_ptr(), dy.data_ptr(), dx.numel()) == 0
    y = dy.cpu().numpy()
    assert np.finfo(np.longdouble).nmant >= 63, "extended precision is needed"
    want = np.exp(x.astype(np.longdouble))
    off = np.abs(y[:x.size].astype(np.longdouble) - want) / want
    print("largest error in units of 2^-52:", float(off.max() * 2.0 ** 52))
    assert (off < 2.0 ** -52).all(), float(off.max() * 2.0 ** 52)
    assert (y[:x.size][x == 0] == 1.0).all()
    assert (y[x.size:-1] == 0.0).all() and y[-1] == 0.0           # below -700, and NaN (of which a row is not cut off)
