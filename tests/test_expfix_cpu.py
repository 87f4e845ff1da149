"""The fixed-point softmax weights (csrc/expfix.cuh) compiled for the host, against 64-bit
exponentials: temperatures and logits over all that 32 bits hold."""
import os
import shutil
import subprocess

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LARGEST = float(np.finfo(np.float32).max)

# the few CUDA built-ins that the header uses, from their definitions
RUNTIME = r"""
#include <math.h>
#include <cstdint>
#include <cstring>
#define __device__
#define __forceinline__ inline
template <class To, class From> inline To bits_as(From v) { To t; std::memcpy(&t, &v, 4); return t; }
inline int __float_as_int(float v) { return bits_as<int>(v); }
inline uint32_t __float_as_uint(float v) { return bits_as<uint32_t>(v); }
inline float __uint_as_float(uint32_t v) { return bits_as<float>(v); }
inline float __fdiv_rn(float a, float b) { return a / b; }
inline int __float2int_rn(float v) { return v != v ? 0 : static_cast<int>(nearbyint(v)); }
inline int __mulhi(int a, int b) { return static_cast<int>(static_cast<int64_t>(a) * b >> 32); }

"""
PROGRAM = r"""
#include "expfix.cuh"
#include <cstdio>
int main() {
  float v[3];                       // max, temperature, z
  while (std::fread(v, 4, 3, stdin) == 3) {
    const memspec::WeightScale s = memspec::weight_scale(v[0], v[1]);
    const unsigned long long w = memspec::weight(v[2], s, memspec::exp_table());
    std::fwrite(&w, 8, 1, stdout);
  }
}
"""


@pytest.fixture(scope="module")
def weights(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    d = tmp_path_factory.mktemp("expfix")
    (d / "cuda_runtime.h").write_text(RUNTIME)
    (d / "t.cpp").write_text(PROGRAM)
    csrc = os.path.join(ROOT, "paper_2608_10362_gb300", "csrc")
    subprocess.run([gxx, "-std=c++17", "-O1", "-ffp-contract=off", "-I", str(d), "-I", csrc, str(d / "t.cpp"), "-o",
                    str(d / "t")], check=True)

    def run(top, T, z):
        v = np.stack(np.broadcast_arrays(*(np.asarray(a, np.float32) for a in (top, T, z))), -1)
        out = subprocess.run([str(d / "t")], input=np.ascontiguousarray(v).tobytes(), capture_output=True, check=True)
        return np.frombuffer(out.stdout, np.uint64).reshape(v.shape[:-1])
    return run


def _check(weights, top, T, z):
    """Off by at most 2^-29.9 of the weight and 2^-46 of the largest one (a unit), 0 below 2^-45;
    the exponential in 64 bits by 2^-46 of itself at most (its argument above -32).

    2^-29.9, with 256 (z - max) c = n + f: of z and of the maximum, 256 z c (|256 z c| < 2^22) has a
    first product that is off by 2^-26 (its rest is at most 1/2), plus its lower part (at most
    1/4) by 2^-25; their difference f (at most 1.5) by 2^-24: 5 * 2^-25 together, which is ln 2 / 256
    times that of the weight, 2^-31.2.  The cubic's value is at most 2^-7.9 and its coefficients,
    the inner sums and the last product are off by 2^-25, 2^-24.5 and 2^-24 of it: 2^-30.8."""
    top, T, z = (np.asarray(a, np.float32) for a in (top, T, z))
    got = weights(top, T, z).astype(np.float64)
    with np.errstate(over="ignore", under="ignore", invalid="ignore"):
        want = 2.0 ** 46 * np.exp((z.astype(np.float64) - top.astype(np.float64)) / T.astype(np.float64))
    want = np.where(z == -np.inf, 0.0, want)
    bad = np.abs(got - want) > want * 2.0 ** -29.9 + 1 + 2.0 * (got == 0)
    assert not bad.any(), [tuple(np.broadcast_to(a, bad.shape)[bad][0] for a in (top, T, z, got, want)), bad.sum()]


def test_ordinary_logits(weights):
    rng = np.random.default_rng(1)
    n = 200000
    T = np.exp(rng.uniform(np.log(0.01), np.log(50), n)).astype(np.float32)
    top = rng.normal(size=n).astype(np.float32) * 20
    z = (top - T * rng.uniform(0, 33, n)).astype(np.float32)
    _check(weights, top, T, z)
    _check(weights, top, T, top)


def test_logits_far_from_zero(weights):
    """256 z c as large as the short way takes them, where its roundings are largest."""
    rng = np.random.default_rng(3)
    n = 400000
    T = np.exp(rng.uniform(np.log(0.05), np.log(5), n)).astype(np.float32)
    top = (T * rng.uniform(5000, 12000, n) * rng.choice([-1, 1], n)).astype(np.float32)
    _check(weights, top, T, (top - T * rng.uniform(0, 33, n)).astype(np.float32))


def test_logits_and_temperatures_of_any_size(weights):
    rng = np.random.default_rng(2)
    n = 200000
    T = np.exp2(rng.uniform(-60, 127.9, n)).astype(np.float32)
    top = (np.exp2(rng.uniform(-60, 127.9, n)) * rng.choice([-1, 1], n)).astype(np.float32)
    with np.errstate(over="ignore"):
        z = (top.astype(np.float64) - T.astype(np.float64) * rng.uniform(0, 33, n)).astype(np.float32)
    z = np.maximum(z, -LARGEST).astype(np.float32)
    _check(weights, top, T, z)


@pytest.mark.parametrize("T", [1.0, 1e10, 1e19, 2e19, 1e30, 1e36, 1e37, 3e37, 1e38, 2e38, LARGEST, np.inf])
def test_the_widest_rows(weights, T):
    """Infinities count as the largest finite number, masks are of the type's lowest value: their
    difference is past what 32 bits hold."""
    top = np.array([LARGEST, LARGEST, 1e38, 12.0, 0.0, -1e38, -LARGEST], np.float32)[:, None]
    z = np.array([-np.inf, -LARGEST, -3e38, -1e38, -1e20, -5.0, 0.0, 3.0, 1e20, 1e38, 3e38, LARGEST], np.float32)[None]
    _check(weights, top, T, np.minimum(z, top))
