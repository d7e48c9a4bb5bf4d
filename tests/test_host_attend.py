"""CPU: division by a number known on the host and the slot of a position
(csrc/pcs_attend.h), and the binding's structs against include/pcs.h."""
import ctypes
import os
import shutil
import subprocess

import pytest

from paper_2607_21686_gb300 import build, pcs

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

_CHECK = r"""
#include <cstdio>
#include <cstdlib>
#include "pcs_attend.h"
using namespace pcs;
static unsigned long long seed = 1;
static uint32_t draw() {
  seed = seed * 6364136223846793005ull + 1442695040888963407ull;
  return static_cast<uint32_t>(seed >> 33);
}
int main() {
  const uint32_t few[] = {0, 1, 2, 3, 0x7ffffffe, 0x7fffffff};
  for (int i = 0; i < 20000; ++i) {
    const uint32_t d = i < 300 ? i + 1 : i < 320 ? 0x7fffffffu - (i - 300) : (draw() >> (draw() % 31)) | 1u;
    FastDiv f;
    f.set(d);
    for (uint32_t n : few)
      if (f.div(n) != n / d) { std::printf("%u / %u\n", n, d); return 1; }
    for (int k = 0; k < 50; ++k) {
      const uint32_t n = k & 1 ? draw() : static_cast<uint32_t>((static_cast<uint64_t>(draw() / d) * d + (k & 2 ? d - 1 : 0)) & 0x7fffffff);
      if (f.div(n) != n / d) { std::printf("%u / %u\n", n, d); return 1; }
    }
  }
  for (int sinks = 0; sinks < 5; ++sinks)
    for (int ring = 0; ring < 9; ++ring) {
      CacheDev c = {};
      c.sinks = sinks;
      c.ring_rows = ring;
      if (ring) c.ring.set(ring);
      for (uint32_t p = 0; p < 60; ++p) {
        const uint32_t want = ring == 0 || p < uint32_t(sinks) ? p : sinks + (p - sinks) % ring;
        if (c.slot_of(p) != want) { std::printf("slot of %u\n", p); return 1; }
      }
    }
  std::puts("ok");
}
"""

_LAYOUT = r"""
#include <stddef.h>
#include <stdio.h>
#include "pcs.h"
#define S(T) printf(#T " %zu\n", sizeof(T));
#define O(T, f) printf(#T "." #f " %zu\n", offsetof(T, f));
int main(void) {
  S(pcs_heads) O(pcs_heads, token_stride) O(pcs_heads, head_stride) O(pcs_heads, heads) O(pcs_heads, head_dim) O(pcs_heads, dtype)
  S(pcs_rotary) O(pcs_rotary, freq) O(pcs_rotary, axes) O(pcs_rotary, pairs) O(pcs_rotary, flags)
  S(pcs_kv_cache) O(pcs_kv_cache, v) O(pcs_kv_cache, table) O(pcs_kv_cache, v_table) O(pcs_kv_cache, table_stride)
  O(pcs_kv_cache, page_stride) O(pcs_kv_cache, row_stride) O(pcs_kv_cache, head_stride) O(pcs_kv_cache, n_pages)
  O(pcs_kv_cache, table_pages) O(pcs_kv_cache, page_rows) O(pcs_kv_cache, heads) O(pcs_kv_cache, head_dim)
  O(pcs_kv_cache, sinks) O(pcs_kv_cache, ring) O(pcs_kv_cache, dtype)
  S(pcs_kv_batch) O(pcs_kv_batch, q_off) O(pcs_kv_batch, tokens) O(pcs_kv_batch, sessions) O(pcs_kv_batch, max_new)
  O(pcs_kv_batch, max_len)
  S(pcs_attend_params) O(pcs_attend_params, scale) O(pcs_attend_params, window) O(pcs_attend_params, flags)
  return 0;
}
"""


def test_division_and_slots(tmp_path):
    gxx = shutil.which("g++")
    cuda = os.path.join(build._cuda_home(), "include")
    if not gxx or not os.path.exists(os.path.join(cuda, "cuda_runtime.h")):
        pytest.skip("no g++ or no CUDA headers")
    src, exe = tmp_path / "check.cpp", tmp_path / "check"
    src.write_text(_CHECK)
    subprocess.run([gxx, "-O1", "-std=c++17", "-I", build.CSRC, "-I", build.INCLUDE, "-I", cuda, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert out.stdout.strip() == "ok", out.stdout


def test_binding_structs_match_header(tmp_path):
    gcc = shutil.which("gcc")
    if not gcc:
        pytest.skip("no C compiler")
    src, exe = tmp_path / "layout.c", tmp_path / "layout"
    src.write_text(_LAYOUT)
    subprocess.run([gcc, "-I", build.INCLUDE, str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    seen = 0
    for line in out.splitlines():
        name, value = line.split()
        struct, _, field = name.partition(".")
        t = getattr(pcs, struct)
        got = getattr(t, field).offset if field else ctypes.sizeof(t)
        assert got == int(value), name
        seen += 1
    assert seen > 30
