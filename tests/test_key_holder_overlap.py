"""The key holder's overlap check against brute force over the bytes of small sets of rows."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INCLUDE = "/opt/rocm/include"

PROGRAM = r"""
#include <cstdio>
#include <set>
#include "rows.hpp"
using namespace fiona_host;

static std::set<uint64_t> bytes(const Rows &r) {
  std::set<uint64_t> s;
  for (uint64_t i = 0; i < r.n[0]; ++i)
    for (uint64_t j = 0; j < r.n[1]; ++j)
      for (uint64_t k = 0; k < r.n[2]; ++k)
        for (uint64_t e = 0; e < r.width * r.elem; ++e)
          s.insert((uint64_t)r.base + (i * r.stride[0] + j * r.stride[1] + k * r.stride[2]) * r.elem + e);
  return s;
}
static bool meet(const Rows &a, const Rows &b) {
  const auto x = bytes(a);
  for (uint64_t v : bytes(b))
    if (x.count(v)) return true;
  return false;
}

int main() {
  uint64_t state = 7;
  auto draw = [&](uint32_t n) { return (uint32_t)((state = state * 6364136223846793005u + 1442695040888963407u) >> 33) % n; };
  int wrong = 0, nested = 0, apart = 0;
  auto check = [&](const Rows &a, const Rows &b, bool exact, const char *what) {
    const bool said = may_overlap(a, b), is = meet(a, b);
    apart += !said;
    if ((is && !said) || (exact && said != is))
      if (wrong++ < 10) printf("%s: said %d, is %d\n", what, said, is);
    if (said != may_overlap(b, a) && wrong++ < 10) printf("%s: not symmetric\n", what);
  };
  // Caches of pages, tokens and heads, keys and values side by side at every axis; whole and shifted by some elements.
  for (uint64_t pages : {1, 3})
    for (uint64_t tokens : {1, 4})
      for (uint64_t heads : {1, 2})
        for (uint64_t d : {1, 5})
          for (int level = 0; level < 4; ++level)
            for (int heads_first = 0; heads_first < 2; ++heads_first) {
              // the axes from the outermost in, with the pair of caches at `level`
              uint64_t count[4], stride[4], step = d;
              const int order[4] = {0, heads_first ? 2 : 1, heads_first ? 1 : 2, -1};
              int at = 0;
              for (int i = 0; i < 4; ++i) {
                if (i == level) count[i] = 2;
                else count[i] = order[at] == 0 ? pages : order[at] == 1 ? tokens : heads, ++at;
              }
              for (int i = 3; i >= 0; --i) stride[i] = step, step *= count[i];
              Rows k{(void *)4096, 2, d, {}, {}};
              at = 0;
              for (int i = 0; i < 4; ++i)
                if (i != level) k.n[order[at]] = count[i], k.stride[order[at]] = stride[i], ++at;
              Rows v = k;
              v.base = (void *)(4096 + 2 * stride[level]);
              char what[64];
              snprintf(what, sizeof what, "level %d, %d pages of %d, %d heads", level, (int)pages, (int)tokens, (int)heads);
              if (may_overlap(k, v) && wrong++ < 10) printf("%s: refused\n", what);
              check(k, v, true, what);
              for (int shift = -6; shift <= 6; ++shift) {
                v.base = (void *)(4096 + 2 * stride[level] + 2 * shift);
                check(k, v, true, what);
              }
            }
  // Sets that nest, over the same steps, anywhere: exact.
  for (int i = 0; i < 20000; ++i) {
    Rows a{(void *)10000, 1u << draw(3), 1 + draw(4), {}, {}};
    uint64_t step = a.width + draw(4);
    for (int j = 2; j >= 0; --j) a.n[j] = 1 + draw(3), a.stride[j] = step, step = step * a.n[j] + draw(6);
    Rows b = a;
    for (int j = 0; j < 3; ++j) b.n[j] = 1 + draw((uint32_t)a.n[j]);
    b.width = 1 + draw((uint32_t)a.width);
    b.base = (void *)(10000 - 20 + a.elem * draw(20 + 2 * (uint32_t)step));
    check(a, b, true, "nested");
    ++nested;
  }
  // Any sets at all: never apart where a byte is shared.
  for (int i = 0; i < 20000; ++i) {
    Rows r[2];
    for (auto &x : r) {
      x = Rows{(void *)(uint64_t)(5000 + draw(150)), 1u << draw(3), 1 + draw(5), {}, {}};
      for (int j = 0; j < 3; ++j) x.n[j] = draw(4), x.stride[j] = draw(40);
    }
    check(r[0], r[1], false, "any");
  }
  if (apart < 1000) return puts("hardly anything apart"), 1;
  if (wrong) return 1;
  puts("ok");
  return 0;
}
"""


def test_overlaps_are_those_of_the_bytes(tmp_path):
    clang = "/opt/rocm/bin/amdclang++"
    if not os.path.exists(clang):
        pytest.skip("no compiler for the library's host headers")
    (tmp_path / "overlap.cpp").write_text(PROGRAM)
    exe = str(tmp_path / "overlap")
    cc = subprocess.run([clang, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I" + ROCM_INCLUDE, "-I" + os.path.join(ROOT, "include"),
                         "-I" + os.path.join(ROOT, "paper_2609_35352_amd", "csrc"), str(tmp_path / "overlap.cpp"), "-o", exe],
                        capture_output=True, text=True)
    assert cc.returncode == 0, cc.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout.strip() == "ok", run.stdout
