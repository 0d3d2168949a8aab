"""How a call of attention with score modifiers is cut (launch_mod.hpp, compiled for
the host), from the call's own description, and what the kernels can walk over.  No
GPU is needed."""

import ctypes
import itertools
import os
import shutil
import subprocess

import numpy as np
import pytest

import paper_2609_18077_amd as vx

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
CUS, ALL = 256, 1 << 62

SOURCE = r"""
#include "launch_mod.hpp"
using namespace vidax;
static const int32_t there = 0;
static ModCall call(int B, int H, int Hkv, int Lq, int Lk, int causal, int valid, int prefix, int start) {
  ModScore s{};
  s.causal = causal;
  s.kv_valid_len = valid ? &there : nullptr;
  s.prefix_len = prefix ? &there : nullptr;
  s.q_start = start ? &there : nullptr;
  return ModCall{B, H, Hkv, Lq, Lk, 1.0f, s};
}
extern "C" void cut(int B, int H, int Hkv, int Lq, int Lk, int causal, int valid, int prefix, int start, int cus, size_t most,
                    int64_t* o) {
  const ModCall c = call(B, H, Hkv, Lq, Lk, causal, valid, prefix, start);
  const ModSplit f = mod_fwd_split(c, cus, most);
  const ModBwdSplit b = mod_bwd_split(c, cus, most);
  o[0] = mod_own_lengths(c.s);
  o[1] = f.few; o[2] = f.units; o[3] = f.pieces.n; o[4] = f.floats;
  o[5] = b.dq.n; o[6] = b.dkdv.n; o[7] = b.floats;
  o[8] = f.runs; o[9] = b.runs;
  o[10] = mod_launches_fit(B, H, Hkv, Lq, Lk, false, false); o[11] = mod_launches_fit(B, H, Hkv, Lq, Lk, true, true);
}
"""


@pytest.fixture(scope="module")
def cut(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("hipcc is not available")
    d = tmp_path_factory.mktemp("mod_calls")
    src, lib = d / "calls.cpp", d / "libcalls.so"
    src.write_text(SOURCE)
    res = subprocess.run([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++17", "-fPIC", "-shared",
                          "-x", "hip", "-I", os.path.join(ROOT, "paper_2609_18077_amd", "csrc"), str(src), "-o",
                          str(lib)], capture_output=True, text=True, timeout=300)
    assert res.returncode == 0, res.stderr[-4000:]
    f = ctypes.CDLL(str(lib)).cut
    f.argtypes = [ctypes.c_int] * 10 + [ctypes.c_size_t, ctypes.c_void_p]
    f.restype = None

    def call(B, H, Hkv, Lq, Lk, causal, valid, prefix, start, most=ALL):
        out = (ctypes.c_int64 * 12)()
        f(B, H, Hkv, Lq, Lk, causal, valid, prefix, start, CUS, most, out)
        return dict(zip(("own", "few", "units", "fwd", "fwd_floats", "dq", "dkdv", "bwd_floats", "runs", "bwd_runs",
                         "fwd_fits", "bwd_fits"), out))

    return call


def _shapes():
    # the first three took pieces that end at the 64th batch, prefixes alone
    yield from ((65, 32, 8, 600, 600), (96, 16, 4, 2049, 2049), (65, 16, 4, 5000, 5000), (64, 32, 8, 600, 600))
    rng = np.random.default_rng(74)
    for _ in range(400):
        Hkv = int(rng.integers(1, 12))
        yield (int(np.exp(rng.uniform(0, 5.4))), Hkv * int(rng.integers(1, 9)), Hkv, int(np.exp(rng.uniform(3, 9))),
               int(np.exp(rng.uniform(3, 9))))


def test_pieces_only_of_batches_that_the_kernels_walk_over(cut):
    """A lane holds the weight of a batch with lengths of its own, and a workgroup goes over at most 16 times 64 tiles to
    find its piece (launch_mod.hpp, each_part in attn_mod.hpp): valid lengths, prefixes and positions alike."""
    taken = large = 0
    for B, H, Hkv, Lq, Lk in _shapes():
        for causal, valid, prefix, start in itertools.product((0, 1), repeat=4):
            if prefix and not causal:
                continue
            got = cut(B, H, Hkv, Lq, Lk, causal, valid, prefix, start)
            assert got["own"] == (valid or prefix or start)
            for side, L in (("fwd", Lq), ("dq", Lq), ("dkdv", Lk)):
                if not got[side]:
                    continue
                taken += 1
                tiles = -(-L // 256)
                if got["own"]:
                    assert B <= 64, (B, H, Hkv, Lq, Lk, side, valid, prefix, start)
                    assert tiles <= 16 or -(-tiles // 64) * B <= 16
                else:
                    large += B > 64
                    assert tiles <= 4096
    assert taken > 500 and large > 50


def test_a_call_takes_no_more_than_its_workspace(cut):
    """Also where less is given than the call would like."""
    for B, H, Hkv, Lq, Lk in _shapes():
        for s in ((1, 0, 1, 0), (1, 1, 0, 1), (0, 1, 0, 0), (1, 0, 0, 0)):
            got = cut(B, H, Hkv, Lq, Lk, *s)
            for side in ("fwd_floats", "bwd_floats"):
                assert cut(B, H, Hkv, Lq, Lk, *s, most=got[side])[side] == got[side]
            least = cut(B, H, Hkv, Lq, Lk, *s, most=0)
            assert least["fwd_floats"] == 0 and least["fwd"] == least["dq"] == least["dkdv"] == least["units"] == 0


def test_few_rows_take_a_prefix_for_no_length_of_a_cache(cut):
    """Causal tokens at the end of equal caches see all of their keys, with a prefix or without."""
    for B, H, Hkv, Lq, Lk in ((16, 32, 8, 1, 16384), (130, 8, 2, 4, 700), (3, 4, 2, 3, 2100)):
        with_prefix, without = cut(B, H, Hkv, Lq, Lk, 1, 0, 1, 0), cut(B, H, Hkv, Lq, Lk, 1, 0, 0, 0)
        assert without["few"] and all(with_prefix[n] == without[n] for n in ("few", "units", "fwd_floats"))


def test_launches_stay_below_two_to_the_32_threads(cut):
    """Whatever is not refused: tiles in workgroups of 512, few rows, joins and ranges in workgroups of 256."""
    rng = np.random.default_rng(75)
    shapes = [(32000, 33, 1, 1, 20), (131072, 8, 8, 40, 40), (40000, 16, 16, 2, 2), (260000, 33, 1, 1, 1)]
    for _ in range(3000):
        Hkv = int(rng.integers(1, 40))
        shapes.append((int(np.exp(rng.uniform(5, 16.6))), Hkv * int(rng.integers(1, 40)), Hkv, int(np.exp(rng.uniform(0, 6.5))),
                       int(np.exp(rng.uniform(0, 6.5)))))
    small = 2 ** 24 - 1  # workgroups of 256
    fit = refused = 0
    for B, H, Hkv, Lq, Lk in shapes:
        tiles = -(-Lq // 128) - (-Lk // 128)
        if tiles * B * H * 64 >= 2 ** 31 or B * H * Lq >= 2 ** 31:
            continue
        qt, kt = -(-Lq // 256) * B * H, -(-Lk // 256) * B * Hkv
        for s in ((0, 0, 0, 0), (1, 0, 0, 0), (1, 1, 0, 1)):
            got = cut(B, H, Hkv, Lq, Lk, *s)
            what = (B, H, Hkv, Lq, Lk, s, got)
            fit += got["fwd_fits"]
            refused += not got["bwd_fits"]
            if got["fwd_fits"]:
                if got["few"]:
                    assert B * Hkv <= small and (not got["units"] or -(-B * H * Lq // 4) <= small), what
                elif got["fwd"]:
                    assert qt * 16 <= small, what
                else:
                    assert qt * got["runs"] * 512 < 2 ** 32 and (got["runs"] == 1 or -(-B * H * Lq // 16) <= small), what
            else:
                assert qt * 512 >= 2 ** 32, what
            if got["bwd_fits"]:
                assert qt * 16 <= small if got["dq"] else qt * 512 < 2 ** 32, what
                assert kt * 32 <= small if got["dkdv"] else kt * got["bwd_runs"] * 512 < 2 ** 32, what
                assert B * (-(-Lq // 64) - (-Lk // 64)) <= 4 * small, what
    assert fit > 1000 and refused > 10


def test_calls_of_too_many_tiles_are_refused():
    P, UNS = 1 << 40, 2
    p = [ctypes.c_void_p(i * P) for i in range(1, 11)]
    for n in ((260000, 33, 1, 1, 1), (1 << 23, 1, 1, 33, 1)):
        assert vx.lib().vidax_attn_mod_fwd(*p[:4], None, *n, 128, 0.1, None, None, 0, None) == UNS
    for n in ((260000, 33, 1, 1, 1), (1 << 23, 1, 1, 1, 1), (1 << 22, 2, 2, 1, 33)):
        assert vx.lib().vidax_attn_mod_bwd(*p[:9], *n, 128, 0.1, None, p[9], 1 << 40, None) == UNS
        assert vx.lib().vidax_attn_mod_bwd_workspace_floats(*n, 128, 0) == 0
    # single tokens of as many requests: a workgroup a K/V head
    assert vx.lib().vidax_attn_mod_fwd_workspace_floats(1 << 22, 2, 2, 1, 33, 128, 1) > 0
