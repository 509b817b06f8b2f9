"""Host check of what the weight gradient's blocks may read: the byte ranges of
``csrc/weight_plan.h`` (which the kernels use, compiled here with g++ on its own)
over every tile, group of columns and step of a plan, against the matrices' ends."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include <stdio.h>
#include <stdlib.h>
#include "weight_plan.h"
using namespace emb;
// the first byte past what may be read of `rows` rows ld bytes apart, of which the last has `row` bytes
static int64_t end_of(int64_t rows, int64_t ld, int64_t row) { return (rows - 1) * ld + row; }
static long fails = 0;
static void range(const char* what, int64_t at, int bytes, int64_t end, bool real, int64_t N, int K, int F) {
  // nothing past the end; where there are columns and rows, everything up to it
  if ((bytes > 0 && at + bytes > end) || (real && at + bytes != end) || bytes < 0) {
    if (++fails < 20) printf("%s N=%lld K=%d F=%d: %lld + %d, end %lld\n", what, (long long)N, K, F, (long long)at, bytes,
                             (long long)end);
  }
}
int main(int argc, char** argv) {
  long large = 0, narrow = 0;
  const int Ns[] = {1, 63, 64, 65, 2048, 4096, 8192, 8191, 32768, 65536, 131072};
  const int Cs[] = {1, 7, 31, 32, 33, 64, 95, 96, 97, 100, 127, 128, 129, 160, 224, 256, 257, 300, 384, 511, 1000, 2048, 4640,
                    5400, 11008, 12800, 40000};
  for (int N : Ns)
    for (int K : Cs)
      for (int F : Cs)
        for (int kind = 0; kind < 3; ++kind) {  // dy: bf16 by words, bf16 by values, fp32
          const int size = kind == 2 ? 4 : 2;
          const bool words = kind != 1;
          const Plan p = plan_for(N, K, F, kind != 0);
          const int tile = p.groups * kGroup;
          if (p.groups == 2) ++large, narrow += K <= 96 || F <= 96;
          const int64_t codes = (K + 31) / 32 * 32, exps = (K + 31) / 32, ld_dy = words ? (F * size + 3) / 4 * 4 : F * size;
          const int64_t row_dy = words ? ld_dy : F * size;
          // the last steps of a part are followed by one more that is loaded ahead
          for (int part = 0; part < p.parts; part = part + 1 < p.parts ? p.parts - 1 : p.parts) {
            const int64_t r1 = (int64_t)(part + 1) * p.steps * kStep;
            for (int64_t r0 = r1 - 2 * kStep; r0 <= r1 + kStep; r0 += kStep) {
              if (r0 < 0) continue;
              const int left = step_rows(N, r0);
              const int64_t rows = left > 0 ? r0 + left : 0;
              for (int k0 = 0; k0 < (K + tile - 1) / tile * tile; k0 += kGroup) {
                const int groups = groups_left(K, k0);
                const bool real = left > 0 && k0 < K;
                range("codes", r0 * codes + k0, rows_bytes(left, (int)codes, groups * 32), end_of(rows, codes, codes), real, N, K, F);
                range("exps", r0 * exps + k0 / 32, rows_bytes(left, (int)exps, groups), end_of(rows, exps, exps), real, N, K, F);
              }
              for (int c0 = 0; c0 < (F + tile - 1) / tile * tile; c0 += kGroup)
                range("dy", r0 * ld_dy + (int64_t)c0 * size, rows_bytes(left, (int)ld_dy, dy_row_bytes(F, c0, size, words)),
                      end_of(rows, ld_dy, row_dy), left > 0 && c0 < F, N, K, F);
            }
          }
        }
  printf("large %ld narrow %ld fails %ld\n", large, narrow, fails);
  return fails ? 1 : large > 100 && narrow > 10 ? 0 : 2;
}
"""


def test_no_block_of_a_weight_gradient_reads_past_its_inputs(tmp_path):
    src, exe = tmp_path / "t.cpp", tmp_path / "t"
    src.write_text(PROGRAM)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-I", os.path.join(ROOT, "paper_2112_02752_amd", "csrc"),
                           "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)])
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout[-3000:]
