"""2^x by additions and products, as the attention over tiles takes every fourth pair of its exponentials: compiled into a small library of its
own and compared with 2^x in 64 bits.  (The attention's tolerances, half steps of 16-bit weights, would not see it lose nine bits.)"""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest
import torch

from conftest import ROOT
from paper_2607_21042_b200 import build

pytestmark = pytest.mark.gpu

PROGRAM = r"""
#include <algorithm>
#include "attention_tiles.cuh"
__global__ void both(const float *x, float *y, int pairs) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i >= pairs) return;
  float a, b;
  ttsgpt::unpack_f32x2(ttsgpt::poly_exp2(ttsgpt::pack_f32x2(x[2 * i], x[2 * i + 1])), a, b);
  y[2 * i] = a; y[2 * i + 1] = b;
}
extern "C" int run(const float *x, float *y, int pairs, void *stream) {
  both<<<(pairs + 255) / 256, 256, 0, (cudaStream_t)stream>>>(x, y, pairs);
  return (int)cudaGetLastError();
}
"""


@pytest.fixture(scope="module")
def poly(tmp_path_factory):
    d = tmp_path_factory.mktemp("poly")
    (d / "p.cu").write_text(PROGRAM)
    subprocess.run([build.nvcc_path(), "-std=c++17", "-O3", "-shared", "-Xcompiler", "-fPIC", "-gencode", "arch=compute_100a,code=sm_100a",
                    "-I", os.path.join(ROOT, "paper_2607_21042_b200", "csrc"), "-o", str(d / "p.so"), str(d / "p.cu")], check=True)
    lib = C.CDLL(str(d / "p.so"))
    lib.run.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p]

    def call(x):
        x = torch.as_tensor(np.asarray(x, np.float32)).to("cuda:0")
        assert x.numel() % 2 == 0
        y = torch.empty_like(x)
        assert lib.run(x.data_ptr(), y.data_ptr(), x.numel() // 2, torch.cuda.current_stream().cuda_stream) == 0
        return y.cpu().numpy()
    return call


def test_relative_error(poly):
    """At most 2^-22, the error of the special-function unit's 2^x beside it, wherever the result is a normal number."""
    rng = np.random.default_rng(0)
    x = np.concatenate([np.linspace(-126, 127, 1 << 20), np.linspace(-1, 1, 1 << 20), rng.uniform(-20, 8, 1 << 20), np.arange(-126, 128), np.arange(-126, 127) + 0.5,
                        np.nextafter(np.float32(np.arange(-125, 127) + 0.5), np.float32(200)), [0.0]]).astype(np.float32)
    x = x[:x.size // 2 * 2]
    y, want = poly(x).astype(np.float64), np.exp2(x.astype(np.float64))
    assert np.max(np.abs(y - want) / want) <= 2.0 ** -22


def test_small_values_and_what_is_not_a_number(poly):
    x = np.array([-126.25, -126.5, -127.0, -127.5, -1000.0, -3e38, -np.inf, -np.inf], np.float32)
    y = poly(x)
    assert np.all(y >= 0) and np.all(y <= 2.0 ** -126) and np.all(y[2:] == 0)
    y = poly(np.array([np.nan, 1.0, 2.0, np.nan], np.float32))
    assert np.isnan(y[0]) and np.isnan(y[3]) and abs(y[1] - 2) <= 2.0 ** -21 and abs(y[2] - 4) <= 2.0 ** -20
