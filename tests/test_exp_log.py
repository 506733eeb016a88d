"""The kernels' 64-bit exponential (csrc/slim_exp.cuh), compiled for the host, against extended precision (CPU)."""
import ctypes
import os
import subprocess

import numpy as np
import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_14917_b200", "csrc")


@pytest.fixture(scope="module")
def exp_log(tmp_path_factory):
    d = tmp_path_factory.mktemp("exp")
    src, so = d / "e.cpp", d / "e.so"
    src.write_text('#include "slim_exp.cuh"\nextern "C" void run(const double* x, double* y, long n) { for (long i = 0; i < n; ++i) y[i] = slim::exp_log(x[i]); }\n')
    subprocess.run([os.environ.get("CXX", "g++"), "-O2", "-std=c++17", "-fPIC", "-shared", "-I" + CSRC, str(src), "-o", str(so)], check=True)
    lib = ctypes.CDLL(str(so))

    def run(x):
        x = np.ascontiguousarray(x, np.float64)
        y = np.empty_like(x)
        lib.run(x.ctypes.data_as(ctypes.c_void_p), y.ctypes.data_as(ctypes.c_void_p), ctypes.c_long(x.size))
        return y
    return run


def test_within_its_bound(exp_log):
    if np.finfo(np.longdouble).nmant < 63:
        pytest.skip("no extended precision on this host")
    rng = np.random.default_rng(0)
    halves = (np.arange(-1009, 116) + 0.5) * np.log(2.0)                     # where the reduced argument is largest
    x = np.concatenate([rng.uniform(-700, 80, 400000), rng.uniform(-2, 2, 200000), -np.exp(rng.uniform(-40, 6.5, 200000)), halves, np.nextafter(halves, 0),
                        [0.0, -0.0, -700.0, 80.0, -5e-324]])
    want = np.exp(x.astype(np.longdouble))
    err = np.abs((exp_log(x) - want) / want)
    assert err.max() < 1e-14, float(err.max())


def test_ends(exp_log):
    y = exp_log([-np.inf, -700.0000001, -1e300, np.nan, 0.0, 80.5, 1e4, np.inf])
    assert (y[:3] == 0).all() and np.isnan(y[3]) and y[4] == 1.0
    assert abs(y[5] / np.exp(80.5) - 1) < 1e-15 and np.isinf(y[6:]).all()
