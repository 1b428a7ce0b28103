"""The host code of the rollout entry points (validation, size arithmetic,
layout, the launch sequence up to the first HIP call) under AddressSanitizer and
UndefinedBehaviorSanitizer, run without a GPU.  The sanitizers apply to host code
only (each flag behind -Xarch_host)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HIPCC = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"

HOST = r"""
#include <climits>
#include <cmath>
#include <cstdint>
#include <cstdio>
#include <initializer_list>
#include "specverify_rollout.h"
static int failures = 0;
static void expect(int line, int got, int want) {
  if (got != want) { std::printf("line %d: %d, expected %d\n", line, got, want); ++failures; }
}
#define EXPECT(call, want) expect(__LINE__, static_cast<int>(call), want)
int main() {
  void* const P = reinterpret_cast<void*>(uintptr_t{1} << 20);
  int32_t* const I = static_cast<int32_t*>(P);
  float* const F = static_cast<float*>(P);
  const int v[] = {INT_MIN, -1, 0, 1, 8, 9, 256, 257, 65536, 151936, SPEC_MAX_V, SPEC_MAX_V + 1, INT_MAX};
  const int64_t st[] = {INT64_MIN, -1, 0, 1, int64_t{1} << 40, INT64_MAX};
  for (int dt = -1; dt < 3; ++dt)
    for (int a : v)
      for (int b : v)
        for (int c : v) {
          const spec_dtype d = static_cast<spec_dtype>(dt);
          for (int m : {0, 1, 256, 257})
            if (spec_top_logits_workspace_size(a, b, c, m, d) % 256 || spec_distill_workspace_size(a, b, c, m, d) % 256)
              ++failures;
          if (spec_verify_probs_workspace_size(a, b, c, d) % 256) ++failures;
          // no workspace: nothing is ever launched
          for (int64_t s : st) {
            if (spec_top_logits(P, s, s, d, a, b, c, 4, nullptr, 1.f, I, F, F, nullptr, 0, nullptr) == SPEC_OK) ++failures;
            if (spec_distill_loss_fwd_bwd(P, s, s, d, a, b, c, I, F, s, s, 4, F, s, s, 1.f, SPEC_DISTILL_CE, 1.f, F, F,
                                          P, SPEC_F32, nullptr, 0, nullptr) == SPEC_OK) ++failures;
            if (spec_verify_probs(P, s, s, P, s, s, d, a, b, c, I, F, F, I, I, I, F, nullptr, 0, nullptr) == SPEC_OK)
              ++failures;
          }
        }
  // valid calls without a device: laid out, then the launch fails
  const size_t big = size_t{1} << 34;
  for (float T : {1e-45f, 1e-38f, 0.7f, 1.f, 3e38f})
    EXPECT(spec_distill_loss_fwd_bwd(P, 300, 100, SPEC_BF16, 4, 3, 100, I, F, 24, 8, 8, F, 3, 1, T, SPEC_DISTILL_FORWARD,
                                     1.f, F, F, P, SPEC_BF16, P, big, nullptr), SPEC_EHIP);
  for (int N : {1, 4, 1000}) {
    EXPECT(spec_top_logits(P, 300, 100, SPEC_BF16, N, 3, 100, 8, F, 1.f, I, F, F, P, big, nullptr), SPEC_EHIP);
    EXPECT(spec_top_logits(P, 1 << 20, 1 << 18, SPEC_F32, N, 3, 151937, 8, nullptr, 1.f, I, F, nullptr, P, big, nullptr),
           SPEC_EHIP);
    EXPECT(spec_verify_probs(P, 400, 100, nullptr, 0, 0, SPEC_F32, N, 3, 100, I, F, F, nullptr, I, I, F, P, big, nullptr),
           SPEC_EHIP);
    EXPECT(spec_verify_probs(P, 100, 100, nullptr, 0, 0, SPEC_BF16, N, 0, 100, nullptr, nullptr, F, I, I, I, nullptr, P,
                             big, nullptr), SPEC_EHIP);
  }
  std::printf("%d failures\n", failures);
  return failures != 0;
}
"""


@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc is needed to build the library")
def test_host_code_under_sanitizers(tmp_path):
    san = ["-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-Xarch_host",
           "-fno-sanitize-recover=undefined"]
    csrc = os.path.join(ROOT, "paper_2606_12370_amd", "csrc")
    common = ["-O1", "-g", "-std=c++17", *san, "-I" + os.path.join(ROOT, "include")]
    (tmp_path / "h.cpp").write_text(HOST)
    for cmd in ([HIPCC, "--offload-arch=gfx950", *common, "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
                 "-I" + csrc, "-c", os.path.join(csrc, "rollout.hip"), "-o", str(tmp_path / "r.o")],
                [HIPCC, "-x", "c++", *common, "-c", str(tmp_path / "h.cpp"), "-o", str(tmp_path / "h.o")],
                [HIPCC, "--offload-arch=gfx950", *san, str(tmp_path / "r.o"), str(tmp_path / "h.o"), "-o",
                 str(tmp_path / "h")]):
        r = subprocess.run(cmd, capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stderr[-3000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1", HIP_VISIBLE_DEVICES="")
    r = subprocess.run([str(tmp_path / "h")], capture_output=True, text=True, timeout=300, env=env)
    out = r.stdout + r.stderr
    assert "runtime error" not in out and "AddressSanitizer" not in out and r.returncode == 0, out[-4000:]
    assert "0 failures" in r.stdout.splitlines()
