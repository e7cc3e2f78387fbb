"""Calls of the recurrent operators over more workgroups than a launch takes (csrc/eql_slices.h, conv_place of csrc/eql_conv.h),
on the CPU: the slices and the place of every workgroup and thread, compiled for the host, with launches of a few
workgroups.  Every strip of every sequence's columns is taken exactly once, and nothing else is touched."""
import ctypes
import os
import subprocess

import pytest

from paper_2607_21271_amd import _lib

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2607_21271_amd", "csrc")
HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

DRIVER = r'''
#include "eql_conv.h"
#include "eql_slices.h"
using namespace eqk;

// hits[b * L * CT ..]: how often a thread owns the token's column; the number of places outside the call
template <int VEC, int MODE>
static long conv(const ConvArgs& a, int64_t most, int64_t reach, int* hits) {
  long outside = 0;
  slices(a.B, a.groups * a.cblocks, most, reach, [&](int64_t seq, unsigned first, unsigned blocks) {
    ConvArgs s = a;
    s.seq = seq;
    s.first = first;
    for (unsigned block = 0; block < blocks; ++block)
      for (int thread = 0; thread < 256; ++thread) {
        const ConvPlace p = conv_place<VEC, MODE>(s, block, thread);
        if (p.b < 0 || p.b >= a.B || p.group < 0 || p.group >= a.groups) {
          ++outside;
          continue;
        }
        for (int64_t l = p.l0; l < p.l1; ++l)
          for (int i = p.skip; i < p.n; ++i) {
            if (p.col + i >= a.CT || l >= a.L) ++outside;
            else ++hits[(p.b * a.L + l) * a.CT + p.col + i];
          }
      }
    return true;
  });
  return outside;
}
extern "C" long conv_places(int64_t B, int64_t L, int C, int T, int W, int dt, int back, int mode, int64_t most, int64_t reach,
                            int* hits) {
  ConvArgs a{};
  a.B = B;
  a.L = L;
  a.C = C;
  a.T = T;
  a.W = W;
  conv_plan(a, dt, 256, back);
  const int vec = conv_vec(dt, W, back);
  if (vec == 8) return mode == 0 ? conv<8, kWhole>(a, most, reach, hits) : mode == 1 ? conv<8, kLoose>(a, most, reach, hits) : conv<8, kTiny>(a, most, reach, hits);
  return mode == 0 ? conv<4, kWhole>(a, most, reach, hits) : mode == 1 ? conv<4, kLoose>(a, most, reach, hits) : conv<4, kTiny>(a, most, reach, hits);
}
// hits[seqs * per]; the most workgroups of a launch
extern "C" int64_t places(int64_t seqs, int64_t per, int64_t most, int64_t reach, int* hits) {
  int64_t largest = 0;
  slices(seqs, per, most, reach, [&](int64_t seq, unsigned first, unsigned blocks) {
    largest = blocks > largest ? blocks : largest;
    for (unsigned block = 0; block < blocks; ++block) {
      const SlicePlace p = slice_place(seq, first, block, (unsigned)per);
      if (p.seq >= 0 && p.seq < seqs) ++hits[p.seq * per + p.at];
    }
    return true;
  });
  return largest;
}
'''


@pytest.fixture(scope="module")
def host(tmp_path_factory):
    if not os.path.exists(HIPCC):
        pytest.skip("needs hipcc")
    d = tmp_path_factory.mktemp("slices")
    (d / "driver.hip").write_text(DRIVER)
    so = str(d / "libslices.so")
    lib = os.path.abspath(_lib.lib()._name)
    obj = str(d / "driver.o")
    for cmd in ([HIPCC, "--offload-arch=gfx950", "--offload-host-only", "-O1", "-std=c++20", "-fPIC", "-I" + CSRC, "-c", str(d / "driver.hip"),
                 "-o", obj], [HIPCC, "-shared", obj, lib, "-Wl,-rpath," + os.path.dirname(lib), "-o", so]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
    h = ctypes.CDLL(so)
    h.conv_places.restype, h.places.restype = ctypes.c_long, ctypes.c_int64
    h.conv_places.argtypes = [ctypes.c_int64] * 2 + [ctypes.c_int] * 6 + [ctypes.c_int64] * 2 + [ctypes.c_void_p]
    h.places.argtypes = [ctypes.c_int64] * 4 + [ctypes.c_void_p]
    return h


WHOLE, LOOSE, TINY = 0, 1, 2


# B, L, C, T, W, mode: one token, several strips, several blocks of columns, rows off the vectors and shorter than one
@pytest.mark.parametrize("size", [(29, 1, 8, 4, 4, WHOLE), (5, 70, 520, 8, 4, WHOLE), (7, 40, 2048, 2, 8, WHOLE), (3, 300, 15, 5, 4, LOOSE),
                                  (11, 33, 2053, 1, 1, LOOSE), (13, 5000, 3, 1, 3, TINY)], ids=lambda s: "x".join(map(str, s)))
@pytest.mark.parametrize("most,reach", [(1, 1 << 12), (7, 1 << 12), (64, 1 << 12), (3, 40), (1 << 24, (1 << 31) - 1)])
@pytest.mark.parametrize("back", [0, 1])
@pytest.mark.parametrize("dt", [_lib.EQL_F32, _lib.EQL_F16])
def test_convolution_takes_every_strip_once(host, size, most, reach, back, dt):
    B, L, C, T, W, mode = size
    hits = (ctypes.c_int * (B * L * C * T))()
    assert host.conv_places(B, L, C, T, W, dt, back, mode, most, reach, hits) == 0
    assert set(hits) == {1}


@pytest.mark.parametrize("seqs,per,most,reach", [(1, 1, 1, 1), (100, 7, 13, 50), (3, 50, 8, 50), (17, 3, 1000, 3), (1000, 1, 7, 64)])
def test_slices_take_every_workgroup_once(host, seqs, per, most, reach):
    hits = (ctypes.c_int * (seqs * per))()
    assert 0 < host.places(seqs, per, most, reach, hits) <= most
    assert set(hits) == {1}
