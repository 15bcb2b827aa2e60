"""How the calls of differential attention split their walks, on the CPU: the
library's host file, its launches replaced by ones that keep what they are given."""
import subprocess

import pytest

from paper_2007_09835_amd import build

PROGRAM = r"""
#include <cstdarg>
#include <cstdio>
#include <cstdlib>
#include <random>
#include "rt3d_tokens.cpp"

namespace rt3d {
rt3d_status fail(rt3d_status s, const char *, ...) { return s; }
rt3d_status ok() { return RT3D_OK; }
AttnArgs fwd, bwd;
BwdPlan plan;
int launch_attn_fwd(const AttnArgs &a, int, int, void *) { return fwd = a, 0; }
int launch_attn_bwd(const AttnArgs &a, const BwdPlan &p, int, void *) { return bwd = a, plan = p, 0; }
int launch_layernorm_fwd(const NormArgs &, int, void *) { return 0; }
int launch_layernorm_bwd(const NormArgs &, int, void *) { return 0; }
int layernorm_bwd_blocks(int64_t) { return 1; }
int launch_rope(const RopeArgs &, int, int, int, void *) { return 0; }
}  // namespace rt3d
extern "C" const char *hipGetErrorString(hipError_t) { return ""; }

int main() {
  std::mt19937 gen(1);
  auto pick = [&](int lo, int hi) { return std::uniform_int_distribution<int>(lo, hi)(gen); };
  auto wide = [&](double hi) { return static_cast<int>(std::exp(std::uniform_real_distribution<double>(0, std::log(hi))(gen))); };
  const int fixed[][8] = {{4, 36, 6656, 16, 4, 128, 0, 49}, {4, 154, 10488, 4, 4, 128, 0, 0}, {6, 69, 4624, 2, 2, 128, 0, 49},
                          {3, 822, 77, 1, 1, 64, 0, 0}};
  int bad = 0, split = 0, tails = 0;
  void *p = reinterpret_cast<void *>(1 << 20);
  float *f = static_cast<float *>(p);
  for (int i = 0; i < COUNT; ++i) {
    rt3d_diffattn_desc d{};
    if (i < 4) {
      const int *x = fixed[i];
      d.n = x[0], d.lq = x[1], d.lk = x[2], d.hq = x[3], d.hk = x[4], d.d = x[5], d.dtype = x[6], d.frame = x[7];
    } else {
      const int frames[] = {0, 0, 1, 7, 49, 196};
      d.n = wide(32), d.hk = 1 << pick(0, 3), d.hq = d.hk << pick(0, 2), d.d = 8 * pick(1, 16), d.dtype = pick(0, 2);
      d.lq = wide(8000), d.lk = pick(0, 1) ? d.lq : wide(60000), d.frame = frames[pick(0, 5)];
    }
    auto show = [&](const char *what, int a, int b) {
      if (++bad < 20)
        std::printf("n %d lq %d lk %d hq %d hk %d d %d dtype %d frame %d: %s %d, %d\n", d.n, d.lq, d.lk, d.hq, d.hk, d.d,
                    d.dtype, d.frame, what, a, b);
    };
    uint64_t bytes = 0;
    if (rt3d_diffattn_fwd_workspace_size(&d, &bytes) != RT3D_OK) return 2;
    auto call = [&](uint64_t n) {
      if (rt3d_diffattn_fwd(&d, p, p, p, f, nullptr, nullptr, p, nullptr, nullptr, n ? p : nullptr, n, nullptr)) std::abort();
      return fwd;
    };
    // the bytes that the size call reports buy the call that it planned, exactly
    const AttnArgs most = call(~0ull), told = call(bytes);
    const uint64_t one = static_cast<uint64_t>(d.n) * d.hq * d.lq * (4 + 4 * d.d) * 4;
    if (most.splits != told.splits || most.span != told.span) show("splits", most.splits, told.splits);
    if (bytes != (most.splits > 1 ? most.splits * one : 0)) show("bytes for splits", most.splits, static_cast<int>(bytes / one));
    // splits are whole tiles, cover the keys and none lies behind them; with less
    // workspace there are fewer, and none passes what it was given
    auto whole = [&](int splits, int span, const char *what) {
      if (splits < 2) return;
      ++split;
      if (span % 64 || static_cast<int64_t>(splits - 1) * span >= d.lk || static_cast<int64_t>(splits) * span < d.lk)
        show(what, splits, span);
      tails += d.lk - (splits - 1) * span < span / 4;
    };
    whole(most.splits, most.span, "spans");
    const AttnArgs less = call(bytes - bytes / 3);
    whole(less.splits, less.span, "spans of less workspace");
    if (less.splits > 1 && less.splits * one > bytes - bytes / 3) show("workspace", less.splits, most.splits);
    if (rt3d_diffattn_bwd_workspace_size(&d, &bytes) != RT3D_OK) return 2;
    if (rt3d_diffattn_bwd(&d, p, p, p, f, nullptr, nullptr, p, p, f, p, p, p, p, f, p, bytes, nullptr)) std::abort();
    whole(plan.dq_splits, plan.dq_span, "spans of dq");
    const uint64_t stats = static_cast<uint64_t>(d.n) * d.hq * d.lq;
    const uint64_t need = (2 + plan.dq_splits) * stats + (plan.dq_splits > 1 ? plan.dq_splits * stats * 2 * d.d : 0) +
                          (plan.dkv_splits > 1 ? static_cast<uint64_t>(plan.dkv_splits) * d.n * d.hk * d.lk * 4 * d.d : 0);
    if (bytes < need * 4 || bytes > need * 4 + 64) show("bytes of the backward call", plan.dq_splits, plan.dkv_splits);
  }
  std::printf("%d wrong; %d splits, %d of them with a tail below a quarter\n", bad, split, tails);
  return bad != 0;
}
"""


def test_the_workspace_that_is_reported_buys_the_splits_that_are_planned(tmp_path):
    src, exe = tmp_path / "plan.cpp", tmp_path / "plan"
    src.write_text(PROGRAM)
    try:
        subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-DCOUNT=20000", "-D__HIP_PLATFORM_AMD__",
                        "-I", build.CSRC, "-I", "/opt/rocm/include", str(src), "-o", str(exe)], check=True,
                       capture_output=True, text=True)
    except subprocess.CalledProcessError as e:
        pytest.fail(e.stderr[-3000:])
    res = subprocess.run([str(exe)], capture_output=True, text=True)
    print(res.stdout[-2000:])
    assert res.returncode == 0, res.stdout[:3000]
