"""Index arithmetic of the cache's kernels on the host, at sizes that no test has the memory for."""
import subprocess

from paper_2505_21036_b200 import build

PROGRAM = """
#include <stdio.h>
#include "rf_cache.cuh"
int main() {
  const int most = 1 << 30;                        // 2^23 columns of 128 tokens
  for (int len : {0, 1, 127, 128, 1000, most - 1, most - 128, most - 300, most / 2}) {
    for (int add : {0, 1, 2, 128, 300, most / 2, most}) {
      if ((long long)len + add > most) continue;
      for (int M : {add > 0 ? add : 1, most}) {
        const long long grid = ((long long)M - 1 + kPage - 1) / kPage + 1;
        long long wanted = add == 0 ? 0 : ((long long)len + add + kPage - 1) / kPage - len / kPage, got = 0;
        for (long long x = 0; x < grid; x += x < 100 || x + 100 > grid ? 1 : x + 50000 > grid ? 1 : 40000) {
          const int page = rf_append_page(len, add, (unsigned)x);
          const bool in = x < wanted;
          if (in != (page >= 0) || (in && page != len / kPage + x)) { printf("len %d add %d x %lld: %d\\n", len, add, x, page); return 1; }
          got += in;
        }
        if (grid < wanted) { printf("grid of %lld CTAs for %lld pages\\n", grid, wanted); return 1; }
      }
    }
  }
  puts("fine");
}
"""


def test_pages_of_an_append(tmp_path):
    src, exe = tmp_path / "pages.cu", tmp_path / "pages"
    src.write_text(PROGRAM)
    subprocess.run([build.nvcc_path(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout
