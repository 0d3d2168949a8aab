"""Launch shapes of the block norm (launch_block.hpp, compiled for the host): every
token and channel has its lane, and a launch stays below 2^32 threads or the call is
refused.  No GPU is needed."""

import ctypes
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2609_18077_amd as vx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
P, UNS = 1 << 44, 2  # fake device addresses, far apart, never dereferenced

SOURCE = r"""
#include "launch_block.hpp"
using namespace vidax;
extern "C" void shape(int backward, int B, int L, int C, int64_t* o) {
  const BlockShape s = backward ? block_bwd_shape(B, L, C) : block_fwd_shape(B, L, C);
  o[0] = s.chunks; o[1] = s.waves; o[2] = s.groups; o[3] = s.rows; o[4] = s.runs; o[5] = block_launch_fits(s, B);
}
"""


@pytest.fixture(scope="module")
def shape(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc is not available")
    d = tmp_path_factory.mktemp("block_rules")
    src, lib = d / "rules.cpp", d / "librules.so"
    src.write_text(SOURCE)
    res = subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-shared",
                          "-x", "hip", "-I", os.path.join(ROOT, "paper_2609_18077_amd", "csrc"), str(src), "-o",
                          str(lib)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-4000:]
    f = ctypes.CDLL(str(lib)).shape
    f.argtypes = [ctypes.c_int] * 4 + [ctypes.c_void_p]
    f.restype = None

    def call(*a):
        out = (ctypes.c_int64 * 6)()
        f(*a, out)
        return list(out)

    return call


def test_rows_channels_and_threads(shape):
    rng = np.random.default_rng(76)
    refused = 0
    for i in range(4000):
        C = 8 * int(rng.integers(1, 2049))
        tokens = int(np.exp(rng.uniform(0, 21.4)))
        B = int(np.exp(rng.uniform(0, np.log(tokens) + 1e-9))) if i % 3 else tokens
        L = tokens // B
        for backward in (0, 1):
            chunks, waves, groups, rows, runs, fits = shape(backward, B, L, C)
            threads = 64 * waves * groups
            assert waves * 64 * chunks * 8 >= C and (waves - 1) * 64 * 8 < C  # every wave has a channel
            assert threads <= (640 if backward and chunks == 1 else 512) and chunks in ((1, 2, 4) if backward else (1, 2, 3, 4))
            assert (runs - 1) * rows < L <= runs * rows
            assert fits == (B * runs * threads < 2 ** 32)
            assert fits or B * L > 2 ** 22  # as the header says
            refused += not fits
    assert refused > 20


def test_too_many_tokens_are_refused():
    p = [ctypes.c_void_p(i * P) for i in range(1, 7)]
    d = vx.BlockNormDesc(0, 1, 0, 0, 1e-6, 1.0)
    g = vx.BlockNormGrads()
    for B, L, C in ((1 << 24, 1, 64), (1 << 25, 1, 8), ((1 << 31) - 1, 1, 8)):
        assert vx.lib().vidax_block_norm_fwd(p[0], p[1], p[2], p[3], B, L, C, ctypes.byref(d), None) == UNS
        assert vx.lib().vidax_block_norm_bwd(*p, ctypes.byref(g), None, 0, B, L, C, ctypes.byref(d), None) == UNS
        assert vx.lib().vidax_block_norm_bwd_workspace_floats(B, L, C) == 0
    for B, L, C in ((1 << 22, 1, 8192), (1, 1 << 22, 16384)):
        assert vx.lib().vidax_block_norm_bwd_workspace_floats(B, L, C) > 0
