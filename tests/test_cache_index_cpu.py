"""Index arithmetic of the cache's kernels on the host, at sizes that no test has the memory for."""
import subprocess

import pytest

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


ROWS = """
#include <stdio.h>
#include "rf_cache.cuh"
// The keys that the row at p sees, border by border.
static long long walk(long long causal, long long origin, long long len, long long p) {
  if (p < 0) return 0;
  long long end = origin;
  if (p >= end) end += (p - end) / causal * causal;
  while (end <= p) end += causal;
  return end < len ? end : len;
}
int main() {
  int bad = 0;
  const int ends[] = {0x7fffffff, -0x7fffffff - 1};
  for (int causal : {1, 2, 7, 50, 128, 3600, 1 << 30, 0x7fffffff})
    for (int len : {0, 1, 5, 49, 50, 51, 128, 300, 7200, 1 << 30})
      for (int o = -110; o <= 112; ++o) {
        const int origin = o > 110 ? ends[o - 111] : o < 60 ? o : o == 60 ? len : o == 61 ? len - 1 : o == 62 ? -(1 << 30) : o * 997 % 9000;
        for (int q_len : {1, 50, 60, 301})
          for (int i = 0; i < q_len; i += q_len > 70 ? 37 : 1)
            bad += rf_row_sees(causal, origin, len, q_len, i) != walk(causal, origin, len, (long long)len - q_len + i);
      }
  // the most that any row of a block sees, rows of several heads one behind the other
  for (int M : {1, 2, 3, 50, 127, 130, 300})
    for (int G : {1, 2, 3, 16, 70})
      for (int q_len : {0, 1, M / 2, M - 1, M})
        for (int len : {0, 3, 129, 500})
          for (int causal : {0, 1, 50})
            for (int origin : {0, 17, -33, 140, 1000}) {
              RfQueries u = {M, G, M * G, (M * G + 127) / 128, causal, nullptr, nullptr, nullptr};
              for (int n : {8, 16, 128, 256})
                for (int r0 = 0; r0 < u.rows; r0 += n) {
                  int most = -1;
                  for (int r = r0; r < r0 + n && r < u.rows; ++r)
                    if (r % M < q_len && rf_row_sees(causal, origin, len, q_len, r % M) > most) most = rf_row_sees(causal, origin, len, q_len, r % M);
                  bad += rf_rows_see(u, origin, len, q_len, r0, n) != most;
                }
            }
  if (bad) printf("%d wrong\\n", bad); else puts("fine");
  return bad != 0;
}
"""


@pytest.mark.parametrize("program", [PROGRAM, ROWS], ids=["pages of an append", "keys that rows see"])
def test_index_arithmetic(tmp_path, program):
    src, exe = tmp_path / "probe.cu", tmp_path / "probe"
    src.write_text(program)
    subprocess.run([build.nvcc_path(), "-std=c++17", "-gencode", "arch=compute_100a,code=sm_100a", "-I", build.CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout
