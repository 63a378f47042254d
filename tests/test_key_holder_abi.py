"""The key holder's C entry points without a GPU: the binding packs the header's structs, refusals launch nothing."""
import os
import shutil
import subprocess

import pytest

import paper_2609_35352_amd as fiona

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
ROCM_INCLUDE = "/opt/rocm/include"


def test_layouts_and_refusals_from_c(tmp_path):
    if shutil.which("gcc") is None or not os.path.isdir(ROCM_INCLUDE):
        pytest.skip("gcc or the ROCm headers are missing")
    if not os.path.exists(fiona.LIB_PATH):
        pytest.fail("libfiona.so is not built (run __graft_entry__.build())")
    exe, lib_dir = str(tmp_path / "layout"), os.path.dirname(fiona.LIB_PATH)
    cc = subprocess.run(["gcc", "-std=c99", "-Wall", "-Wextra", "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROOT, "include"),
                         "-I" + ROCM_INCLUDE, os.path.join(ROOT, "tests", "key_holder_layout.c"), "-L" + lib_dir, "-lfiona",
                         "-Wl,-rpath," + lib_dir, "-o", exe], capture_output=True, text=True)
    assert cc.returncode == 0, cc.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout.strip().endswith("ok"), run.stdout + run.stderr
    lines = run.stdout.splitlines()
    packs = [fiona._KV_CACHE, fiona._APPEND_ARGS, fiona._ATTENTION_DESC, fiona._ATTENTION_ARGS, fiona._ADAPTERS_DESC,
             fiona._ADAPTER_ARGS]
    assert [int(v) for v in lines[0].split()[1:]] == [p.size for p in packs]
    # the fields in question, each set alone, land at the header's offsets
    at = {tuple(line.split()[:2]): int(line.split()[2]) for line in lines[1:-1]}
    for (struct, field), (pack, index, count) in {
            ("fiona_kv_cache", "v_head"): (fiona._KV_CACHE, 12, 13),
            ("fiona_append_args", "sin"): (fiona._APPEND_ARGS, 21, 22),
            ("fiona_attention_args", "q"): (fiona._ATTENTION_ARGS, 5, 15),
            ("fiona_attention_args", "lengths"): (fiona._ATTENTION_ARGS, 14, 15),
            ("fiona_adapter_args", "base"): (fiona._ADAPTER_ARGS, 8, 20),
            ("fiona_adapter_args", "dx_row"): (fiona._ADAPTER_ARGS, 19, 20)}.items():
        data = pack.pack(*[(0x0102030405060708 if i == index else 0) for i in range(count)])
        assert data[at[struct, field]:at[struct, field] + 8] == (0x0102030405060708).to_bytes(8, "little"), (struct, field)


PAGES = r"""
#include <cstdio>
#include "rows.hpp"
int main() {
  uint64_t state = 1, wrong = 0;
  auto draw = [&] { return (uint32_t)((state = state * 6364136223846793005u + 1442695040888963407u) >> 33); };   // < 2^31
  auto check = [&](uint32_t size) {
    uint32_t mul, shift;
    fiona_host::page_divisor(size, mul, shift);
    auto page = [&](uint64_t n) {
      if (n >= 1u << 31) return;
      const uint64_t q = mul ? (n * mul >> 32) >> shift : n;
      if (q != n / size && wrong++ < 5) printf("%llu / %u: %llu\\n", (unsigned long long)n, size, (unsigned long long)q);
    };
    for (uint64_t k : {(uint64_t)0, (uint64_t)1, (uint64_t)2, (uint64_t)(0x7fffffffu / size)})
      for (int e = -1; e <= 1; ++e) page(k * size + e);
    for (int i = 0; i < 50; ++i) page(draw());
    page(0x7fffffffu);
  };
  for (uint32_t size = 1; size < 2000; ++size) check(size);
  for (int k = 1; k < 31; ++k) check(1u << k), check((1u << k) + 1), check((1u << k) - 1);
  for (int i = 0; i < 2000; ++i) check(1 + draw() % ((1u << 30) - 1));
  return wrong != 0;
}
"""


def test_page_division_is_exact(tmp_path):
    """The multiplier and shift that divide a token's number by the page size, over the edges of quotients."""
    clang = "/opt/rocm/bin/amdclang++"
    if not os.path.exists(clang):
        pytest.skip("no compiler for the library's host headers")
    (tmp_path / "pages.cpp").write_text(PAGES)
    exe = str(tmp_path / "pages")
    cc = subprocess.run([clang, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I" + ROCM_INCLUDE, "-I" + os.path.join(ROOT, "include"),
                         "-I" + os.path.join(ROOT, "paper_2609_35352_amd", "csrc"), str(tmp_path / "pages.cpp"), "-o", exe],
                        capture_output=True, text=True)
    assert cc.returncode == 0, cc.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0, run.stdout
