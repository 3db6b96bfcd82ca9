"""How quake_attention_shared cuts a call up (CPU, g++): the plan's text, taken from the
source, over sizes up to the documented limits. What a launch carries has to fit: parts of
keys and tiles in 31 bits, as the kernels divide by them; fewer than 2^24 workgroups of 256
threads a launch; all keys of a list in its parts; a workspace in whole 16 bytes."""
import os
import re
import shutil
import subprocess

import pytest

from paper_2412_00408_amd import build

HARNESS = r"""
#include <algorithm>
#include <cinttypes>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <random>
%(constants)s
%(plan)s
static const char* wrong(const SharedShape& s, bool weigh, bool workspace) {
  const SharedPlan p = shared_plan(s, weigh, workspace);
  const int64_t k31 = (int64_t)1 << 31, k24 = 1 << 24, rows = s.sq * s.group();
  const int64_t heads = s.batch * s.kv_heads, items = heads * wide_tiles(rows, p.many);
  if (p.chunk < 1 || p.chunk * (p.many ? 1 : 2) >= k31) return "keys of a sequence's part";
  if (p.gchunk < 1 || p.gchunk * (p.gmany ? 1 : 2) >= k31) return "keys of a prefix's part";
  if (p.tiles >= k31 || p.gtiles >= k31 || p.nsplit >= k31 || p.gsplit >= k31) return "tiles or parts";
  const int64_t psteps = (s.sp + 63) / 64, steps = (s.skv + 63) / 64 + (p.gsplit > 0 ? 0 : psteps);
  if (p.gsplit > 0 && p.gsplit * p.gchunk < psteps) return "a prefix's keys";
  if (p.cut && p.nsplit * p.chunk < steps) return "a sequence's keys";
  if (p.gsplit > 0 && !p.cut) return "parts of a group that nothing joins";
  if (p.items != items || (!p.cut && p.nsplit != 1)) return "tiles";
  if (p.gitems * p.gsplit + items * p.nsplit >= k24) return "workgroups of the tiles";
  if (p.cut) {
    const int64_t joined = p.many ? items * 128 : heads * rows, slots = p.stored ? (s.skv + 1023) / 1024 : 0;
    const int64_t team = 1024 / s.dim / (p.gsplit + p.nsplit <= 16 ? 1 : 8);
    if ((joined + team - 1) / team + heads * slots >= k24) return "workgroups of the join";
  }
  const SharedSpace x = shared_space(s, p, weigh);
  for (int64_t n : {x.part, x.stats, x.scores, x.sums})
    if (n < 0 || n %% 16 != 0) return "the workspace";
  return nullptr;
}
int main() {
  std::mt19937_64 rng(12345);
  const auto upto = [&](double bits) {          // log-uniform, powers of two and their neighbours among them
    const double u = std::uniform_real_distribution<double>(0.0, bits)(rng);
    const int64_t n = (int64_t)__builtin_exp2(rng() %% 3 ? u : (double)(int64_t)u);
    return std::max<int64_t>(0, n + (int64_t)(rng() %% 3) - 1);
  };
  int64_t seen = 0, cut = 0, grouped = 0, stored = 0;
  for (int i = 0; i < 3000000; ++i) {
    SharedShape s{};
    s.groups = std::max<int64_t>(1, upto(18));
    s.batch = s.groups * upto(10);
    s.kv_heads = std::max<int64_t>(1, upto(5));
    s.heads = s.kv_heads * std::max<int64_t>(1, upto(7));
    s.sq = rng() %% 2 ? 1 : upto(18);
    s.sp = rng() %% 4 ? upto(30) : 0;
    s.skv = rng() %% 8 ? upto(30) : 0;
    s.dim = rng() %% 2 ? 64 : 128;
    if (!shared_shape_ok(s)) continue;
    for (int weigh = 0; weigh < 2; ++weigh) {
      if (weigh && (s.skv == 0 || !weigh_shape_ok(s))) continue;
      for (int workspace = weigh; workspace < 2; ++workspace) {
        if (const char* why = wrong(s, weigh, workspace)) {
          std::printf("%%s: batch %%" PRId64 " groups %%" PRId64 " sq %%" PRId64 " sp %%" PRId64 " skv %%" PRId64
                      " heads %%" PRId64 " kv_heads %%" PRId64 " dim %%" PRId64 " weigh %%d workspace %%d\n",
                      why, s.batch, s.groups, s.sq, s.sp, s.skv, s.heads, s.kv_heads, s.dim, weigh, workspace);
          return 1;
        }
        const SharedPlan p = shared_plan(s, weigh, workspace);
        ++seen;
        cut += p.cut;
        grouped += p.gsplit > 0;
        stored += p.stored;
      }
    }
  }
  if (seen > 100000 && cut > 10000 && grouped > 10000 && stored > 1000) std::printf("all fit\n");
  else std::printf("%%" PRId64 " %%" PRId64 " %%" PRId64 " %%" PRId64 "\n", seen, cut, grouped, stored);
}
"""


def _taken(pattern, text):
    found = re.findall(pattern, text, re.S | re.M)
    assert len(found) == 1, (pattern, len(found))
    return found[0]


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_plans_fit_over_the_documented_sizes(tmp_path):
    with open(os.path.join(build.CSRC, "shared.hip")) as f:
        text = f.read()
    constants = [_taken(r"^constexpr int kShWaves[^;]*;", text), _taken(r"^constexpr int kWeighSlots[^;]*;", text),
                 "static constexpr " + _taken(r"^__host__ __device__ constexpr (int64_t score_row.*?})$", text)]
    parts = dict(constants="\n".join(constants),
                 plan=_taken(r"^struct SharedShape.*?(?=^template <int DT, int MODE, int D, bool WEIGH>\nstatic void)", text))
    src, exe = str(tmp_path / "plan.cpp"), str(tmp_path / "plan")
    with open(src, "w") as f:
        f.write(HARNESS % parts)
    r = subprocess.run(["g++", "-std=c++17", "-O2", "-fwrapv", src, "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-3000:]
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and "all fit" in run.stdout, run.stdout[-600:] + run.stderr[-600:]
