"""No C++ exception leaves an entry point of gift_kv.h: refusals while no memory can be had for their messages."""
import os
import subprocess

import pytest

from paper_2608_25431_amd import build, gift
from test_kv_refusals import lib  # noqa: F401

SOURCE = r"""
#include <dlfcn.h>
#include <stdio.h>
#include <stdlib.h>
#include <new>
#include "gift_kv.h"

static bool none = false;  // no more memory
void* operator new(size_t n) {
  void* p = none ? nullptr : malloc(n);
  if (!p) throw std::bad_alloc();
  return p;
}
void operator delete(void* p) noexcept { free(p); }
void operator delete(void* p, size_t) noexcept { free(p); }

int main(int, char** argv) {
  void* so = dlopen(argv[1], RTLD_NOW);
  if (!so) return printf("%s\n", dlerror()), 2;
  auto append = (decltype(&gift_kv_append))dlsym(so, "gift_kv_append");
  auto attend = (decltype(&gift_tree_attention))dlsym(so, "gift_tree_attention");
  auto tables = (decltype(&gift_kv_tables))dlsym(so, "gift_kv_tables");
  gift_paged_kv kv{};  // a null base, strides of 0: refused by the geometry
  gift_kv_format format{};
  gift_tree_attention_args args{};
  gift_kv_rows rows{};
  gift_kv_step step{};
  none = true;
  for (int i = 0; i < 2; i++) {
    const int s[] = {append(&kv, &format, nullptr, 0, nullptr, &rows, nullptr),
                     attend((gift_attention_work)&kv, &kv, &format, &args, nullptr), tables(&step, nullptr)};
    printf("%d %d %d\n", s[0], s[1], s[2]);
  }
  fflush(stdout);
  _Exit(0);
}
"""


@pytest.mark.skipif(not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"), reason="needs the HIP headers")
def test_refusals_without_memory(lib, tmp_path):  # noqa: F811
    (tmp_path / "main.cpp").write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-O1", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(build.ROOT, "include"),
                    "-I", "/opt/rocm/include", str(tmp_path / "main.cpp"), "-ldl", "-o", str(tmp_path / "main")], check=True,
                   timeout=120)
    r = subprocess.run([str(tmp_path / "main"), gift.LIB_PATH], capture_output=True, text=True, timeout=120)
    assert (r.returncode, r.stdout) == (0, f"{gift.E_INVALID} {gift.E_INVALID} {gift.E_INVALID}\n" * 2), r.stdout + r.stderr
