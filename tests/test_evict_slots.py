"""Loops of evict.hip's choice, taken from the source, on the CPU under AddressSanitizer
and UndefinedBehaviorSanitizer (g++), thread by thread. The one that holds a thread's slots,
for rows on both sides of every limit: it has to fill all of them, with the keys that they
should have, and nothing behind them. The one that clears the counts: it has to reach
all of them and stay within each array."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2412_00408_amd import build

SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all"]

HARNESS = r"""
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <algorithm>
#include <vector>
#define __device__
#define __forceinline__ inline
#define __builtin_amdgcn_sched_barrier(x)
using std::min;
static uint32_t as_u(float f) { uint32_t u; std::memcpy(&u, &f, 4); return u; }
%(keys)s
%(sizes)s
template <int THREADS, int HELD>
static void check(int32_t len, int32_t sinks, int32_t recent) {
  std::vector<float> weights(len);          // of the row's own size: a read behind it is seen
  for (int32_t i = 0; i < len; ++i) weights[i] = i %% 7 == 3 ? NAN : std::sin((float)i);
  const float* w = weights.data();
  const int32_t lo = sinks, hi = len - recent;
  constexpr int E = HELD > 0 ? HELD : kEach;
  for (int wave = 0; wave < THREADS / 64; ++wave) {
    const int32_t run = (len + THREADS - 1) / THREADS * 64;
    const int32_t from = wave * run, to = min(from + run, len);
    for (int lane = 0; lane < 64; ++lane)
      for (int32_t at = from; at < std::max(to, from + 1); at += 64 * E) {
        uint32_t u[E];
        std::fill(u, u + E, 0xABABABABu);
%(fetch)s
        fetch(at);
        for (int e = 0; e < E; ++e) {
          const int32_t i = at + 64 * e + lane;
          const uint32_t want = i >= to ? kNever : i < lo || i >= hi ? kAlways : weight_key(w[i]);
          if (u[e] != want) {
            std::printf("%%d slots, wave %%d lane %%d slot %%d\n", len, wave, lane, e);
            std::exit(1);
          }
        }
      }
  }
  std::printf("%%d threads %%d held %%d slots\n", THREADS, HELD, len);
  std::fflush(stdout);
}
int main() {
  for (int32_t n : {1, 2, 63, 64, 65, 300, 4095, 4096}) check<256, kHeld>(n, 0, 0);
  for (int32_t n : {4097, 5000, 16383, 16384}) check<1024, kHeld>(n, 4, 100);
  for (int32_t n : {16385, 22013, 40959, 40960}) check<1024, kHeldLong>(n, 4, 100);
  for (int32_t n : {40961, 70001}) check<1024, 0>(n, 0, 3);
  std::printf("all held\n");
}
"""


def _taken(pattern, text):
    found = re.findall(pattern, text, re.S | re.M)
    assert len(found) == 1, pattern
    return found[0]


CLEAR = r"""
#include <cstdint>
#include <cstdio>
#include <cstring>
%(sizes)s
%(shared)s
static struct { int x; } threadIdx;
template <int THREADS>
static bool check() {
  static ChooseShared<THREADS> sh;
  std::memset((void*)&sh, 0xFF, sizeof sh);
  for (threadIdx.x = 0; threadIdx.x < THREADS; ++threadIdx.x) {
%(clear)s
  }
  for (int i = 0; i < 3; ++i) {
    static uint32_t none[kBins];
    if (std::memcmp((const char*)&sh.bins + 4 * kBins * i, none, sizeof none) != 0) return false;
  }
  return sh.wave[0] == 0xFFFFFFFFu && sh.found[2] == 0xFFFFFFFFu;
}
int main() {
  if (check<256>() && check<1024>()) std::printf("all clear\n");
}
"""


def _source():
    with open(os.path.join(build.CSRC, "evict.hip")) as f:
        return f.read()


def _taken(pattern, text):
    found = re.findall(pattern, text, re.S | re.M)
    assert len(found) == 1, pattern
    return found[0]


def _runs(tmp_path, code, says):
    src, exe = str(tmp_path / "taken.cpp"), str(tmp_path / "taken")
    with open(src, "w") as f:
        f.write(code)
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", *SAN, src, "-o", exe], capture_output=True, text=True)
    if r.returncode != 0 and "asan" in r.stderr.lower():
        pytest.skip("sanitizer runtime not available: " + r.stderr[-300:])
    assert r.returncode == 0, r.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and says in run.stdout, run.stdout[-600:] + run.stderr[-2000:]


needs_gxx = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
SIZES = r"^constexpr int kBins[^;]*;"


@needs_gxx
def test_held_slots_stay_in_bounds(tmp_path):
    text = _source()
    parts = dict(keys=_taken(r"^constexpr uint32_t kAlways.*?^}$", text), sizes=_taken(SIZES, text),
                 fetch=_taken(r"^  const auto fetch = .*?^  };$", text))
    assert "weight_key" in parts["keys"]
    _runs(tmp_path, HARNESS % parts, "all held")


@needs_gxx
def test_cleared_counts_stay_in_bounds(tmp_path):
    text = _source()
    parts = dict(sizes=_taken(SIZES, text), shared=_taken(r"^template <int THREADS>\nstruct ChooseShared.*?^};$", text),
                 clear=_taken(r"fetch\(from\);\n(.*?)  __syncthreads", text))
    _runs(tmp_path, CLEAR % parts, "all clear")
