"""Numbers at odd addresses are read by aligned words, none of which may reach beyond its matrix: the readers, compiled for the host with
calls at every access to memory, at all addresses, lengths and places."""
import os
import subprocess

from paper_1909_07588_b200 import build

READERS = r"""
#include "laq_ops_gemm.cuh"
using namespace laq::ops;
// eight codes, eight 16-bit numbers and sixteen codes of a matrix's row, as the kernels read them, and what was read
void read(int kind, bool at_once, const uint8_t* row, long long r, long long rows, long long c, long long cols, uint8_t* out) {
  if (kind == 0) {
    const bool edge = at_edge(r, r, rows, c, cols - c - 8, 1);
    const uint2 v = at_once ? load8_any<true>(row + c, (int)(cols - c < 8 ? cols - c : 8), edge) : load8_any(row + c, (int)(cols - c < 8 ? cols - c : 8), edge);
    memcpy(out, &v, 8);
  } else if (kind == 1) {
    const uint16_t* p = reinterpret_cast<const uint16_t*>(row) + c;
    const bool edge = at_edge(r, r, rows, c, cols - c - 8, 2);
    const uint4 v = at_once ? load16_any<true>(p, (int)(cols - c < 8 ? cols - c : 8), edge) : load16_any(p, (int)(cols - c < 8 ? cols - c : 8), edge);
    memcpy(out, &v, 16);
  } else {
    const uint4 v = load16_codes_any(row + c, (int)(cols - c < 16 ? cols - c : 16), at_edge(r, r, rows, c, cols - c - 16, 1));
    memcpy(out, &v, 16);
  }
}
"""

# The callbacks of -fsanitize=thread note every read; nothing of that sanitizer's own library is linked.
MAIN = r"""
#include <cstdint>
#include <cstdio>
#include <cstring>
static const uint8_t *from, *to, *lo, *hi;      // the memory that is watched; the matrix
static int beyond, reads;
static void note(const void* p, int n) {
  const uint8_t* b = (const uint8_t*)p;
  if (b + n <= from || b >= to) return;
  ++reads;
  if (b < lo || b + n > hi) ++beyond;
}
#define SIZED(n) extern "C" void __tsan_read##n(void* p) { note(p, n); } extern "C" void __tsan_unaligned_read##n(void* p) { note(p, n); } \
  extern "C" void __tsan_write##n(void*) {} extern "C" void __tsan_unaligned_write##n(void*) {}
SIZED(1) SIZED(2) SIZED(4) SIZED(8) SIZED(16)
extern "C" void __tsan_read_range(void* p, unsigned long n) { note(p, (int)n); }
extern "C" void __tsan_write_range(void*, unsigned long) {}
extern "C" void __tsan_init() {}
extern "C" void __tsan_func_entry(void*) {}
extern "C" void __tsan_func_exit() {}
extern "C" void* __tsan_memcpy(void* d, const void* s, unsigned long n) { return memcpy(d, s, n); }
void read(int kind, bool at_once, const uint8_t* row, long long r, long long rows, long long c, long long cols, uint8_t* out);
int main() {
  alignas(16) static uint8_t memory[2048];
  for (int i = 0; i < 2048; ++i) memory[i] = (uint8_t)(i * 37 + 11);
  from = memory, to = memory + 2048;
  int wrong = 0, cases = 0;
  for (int kind = 0; kind < 3; ++kind)
    for (int at = 0; at < 16; at += kind == 1 ? 2 : 1)
      for (int cols = 1; cols < 70; ++cols) {
        const int size = kind == 1 ? 2 : 1, step = kind == 2 ? 16 : 8, rows = 1 + cols % 4, ld = cols + at % 4;
        lo = memory + 64 + at, hi = lo + ((rows - 1) * ld + cols) * size;
        for (int r = 0; r < rows; ++r)
          for (int c = 0; c < cols; c += step, ++cases) {
            const uint8_t* row = lo + r * ld * size;
            uint8_t got[16];
            const int n = (cols - c < step ? cols - c : step) * size;
            read(kind, r % 2, row, r, rows, c, cols, got);
            if (memcmp(got, row + c * size, n)) ++wrong;
          }
      }
  printf("%d %d %d %d\n", cases, reads, wrong, beyond);
}
"""


def test_no_word_beyond_a_matrix(tmp_path):
    (tmp_path / "readers.cu").write_text(READERS)
    (tmp_path / "main.cpp").write_text(MAIN)
    flags = [f for f in build.NVCC_FLAGS if f not in ("-shared", "-O3", "-lineinfo")]
    subprocess.run([os.environ.get("NVCC", "nvcc")] + flags + ["-O1", "-Xcompiler", "-fsanitize=thread", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    "-c", "-o", str(tmp_path / "readers.o"), str(tmp_path / "readers.cu")], check=True, capture_output=True)
    subprocess.run([os.environ.get("NVCC", "nvcc"), "-cudart", "static", "-o", str(tmp_path / "reads"), str(tmp_path / "main.cpp"), str(tmp_path / "readers.o"), "-lcuda"],
                   check=True, capture_output=True)
    cases, reads, wrong, beyond = map(int, subprocess.run([str(tmp_path / "reads")], check=True, capture_output=True, text=True).stdout.split())
    assert cases > 10000 and reads > cases and wrong == 0 and beyond == 0
