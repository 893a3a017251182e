"""Row arithmetic of the sequence operators at their limits, compiled for the
host from the header that the kernels include (csrc/seq_index.h).  Signed
overflow wraps here as it does on the GPU."""
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_1908_06649_gb300", "csrc")
MOST_ROWS = 2 ** 31 - 4097


@pytest.fixture(scope="module")
def run(tmp_path_factory):
    folder = tmp_path_factory.mktemp("index")

    def compiled(body):
        src, exe = folder / "p.cpp", folder / "p"
        src.write_text('#include <stdio.h>\n#include <stdlib.h>\n#include "seq_index.h"\n'
                       "using namespace tcu::seq;\n" + body)
        subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-Wall", "-Werror", "-I", CSRC,
                        str(src), "-o", str(exe)], check=True)
        return lambda *args: subprocess.run([str(exe), *map(str, args)], capture_output=True,
                                            text=True)
    return compiled


CHUNKS = r"""
// chunks as the launch splits rows: of 32-row tiles, as even as they go
int main(int, char **argv) {
  const int rows = atoi(argv[1]), tiles = (int)(((int64_t)rows + 31) / 32);
  for (int chunks = 1; chunks <= 1300 && chunks <= tiles; ++chunks) {
    const int64_t each = ((int64_t)tiles + chunks - 1) / chunks * 32, count = (rows + each - 1) / each;
    int64_t seen = 0;
    for (int k = 0; k < count; ++k) {
      const int r0 = (int)(k * each), r1 = chunk_end(r0, (int)each, rows);
      if (r0 != seen || r1 <= r0 || r1 > rows || (k + 1 < count && r1 - r0 != each)) {
        printf("%d chunks: chunk %d is [%d, %d)\n", chunks, k, r0, r1);
        return 1;
      }
      seen = r1;
    }
    if (seen != rows) return 2;
  }
  return 0;
}
"""


@pytest.mark.parametrize("rows", [1, 31, 33, 5000, 2 ** 30 + 1, MOST_ROWS - 31, MOST_ROWS])
def test_chunks_cover_the_rows(run, rows):
    out = run(CHUNKS)(rows)
    assert out.returncode == 0, out


SEQUENCES = r"""
#include <sys/mman.h>
// `count` sequences, all empty but the last, which holds every row.  Pages that
// stay untouched read as zeros.
int main(int, char **argv) {
  const int count = atoi(argv[1]), rows = 100;
  const size_t bytes = ((size_t)count + 1) * 4;
  void *mem = mmap(nullptr, bytes, PROT_READ | PROT_WRITE,
                   MAP_PRIVATE | MAP_ANONYMOUS | MAP_NORESERVE, -1, 0);
  if (mem == MAP_FAILED) return 3;
  int32_t *offsets = (int32_t *)mem;
  offsets[count] = rows;
  for (int t = 0; t < rows; ++t)
    if (sequence_of(offsets, count, t) != count - 1) return 1;
  return sequence_of(offsets, count, 100) == -1 ? 0 : 2;
}
"""


@pytest.mark.parametrize("count", [1, 2, 1000, 2 ** 30 + 5, 2 ** 31 - 1])
def test_sequence_of_a_row_among_many(run, count):
    out = run(SEQUENCES)(count)
    assert out.returncode == 0, out


ORDERS = r"""
int main() {
  const int32_t o[] = {0, 0, 3, 3, 7, 7};  // sequences 1 and 3 hold rows
  const int want[] = {1, 1, 1, 3, 3, 3, 3, -1};
  for (int t = 0; t < 8; ++t)
    if (sequence_of(o, 5, t) != want[t]) return 1;
  if (sequence_of(o, 0, 0) != -1) return 2;
  const int32_t odd[] = {50, 10, 50, -5, 200};
  for (int t = 0; t < 300; ++t)
    if (sequence_of(odd, 4, t) < -1 || sequence_of(odd, 4, t) > 3) return 3;
  return 0;
}
"""


def test_sequence_of_a_row(run):
    out = run(ORDERS)()
    assert out.returncode == 0, out
