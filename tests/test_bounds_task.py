"""How the tasks of the page bounds are split, at the limits of what the call takes: compiled for the CPU, since a task
that is split wrong reads in front of the page table and writes outside the bounds."""
import shutil
import subprocess
from pathlib import Path

import pytest

from test_kernel_sources import functions

CSRC = Path(__file__).resolve().parents[1] / "paper_2606_01790_gb300" / "csrc"

PROBE = r"""
#define __host__
#define __device__
#define __forceinline__ inline
#include <cstdio>
#include <cstdlib>
#include "bounds_task.cuh"

// argv: n, tokens, shift, max_pages, layers, G; the pages, then every task looked at as its number and its four parts
int main(int, char** a) {
  const int n = atoi(a[1]), tokens = atoi(a[2]), shift = atoi(a[3]), max_pages = atoi(a[4]), layers = atoi(a[5]), G = atoi(a[6]);
  const int pages = starkv::bounds_pages(tokens, shift, max_pages);
  printf("%d\n", pages);
  const int64_t each = int64_t(pages) * layers * G, all = each * n;
  const int64_t marks[] = {0, each, each * (n - 1), int64_t(1) << 31, int64_t(1) << 32, int64_t(pages) * G, all - 1, all / 3, all / 7 * 5};
  for (int64_t m : marks)
    for (int64_t t = m - 2; t < m + 3; ++t)
      if (t >= 0 && t < all) {
        const starkv::BoundsTask b(t, pages, layers, G);
        printf("%lld %d %d %d %d\n", static_cast<long long>(t), b.seq, b.layer, b.page, b.g);
      }
  return 0;
}
"""


@pytest.fixture(scope="module")
def probe(tmp_path_factory):
    cc = shutil.which("g++")
    if cc is None:
        pytest.skip("no C++ compiler")
    at = tmp_path_factory.mktemp("bounds_task")
    (at / "probe.cc").write_text(PROBE)
    subprocess.run([cc, "-std=c++17", "-Wall", "-Werror", "-fsanitize=undefined", "-fno-sanitize-recover", f"-I{CSRC}",
                    str(at / "probe.cc"), "-o", str(at / "probe")], check=True)
    return at / "probe"


@pytest.mark.parametrize("n,tokens,shift,max_pages,layers,G", [
    (1, 1, 4, 1, 1, 1), (3, 17, 4, 40, 2, 3), (64, 1, 5, 439, 28, 8), (2, 14032, 6, 220, 28, 4),
    (1, 1 << 24, 4, 1 << 20, 64, 32), (1024, 1 << 24, 4, 1 << 20, 64, 32), (1024, 1 << 24, 4, 1 << 20, 4096, 32),
    (1024, 1 << 24, 8, 1 << 16, 32768, 1), (5, 1 << 24, 4, 3, 100000, 7)])
def test_every_task_is_one_page_of_one_layer_and_head(probe, n, tokens, shift, max_pages, layers, G):
    out = subprocess.run([str(probe), *map(str, (n, tokens, shift, max_pages, layers, G))], check=True, capture_output=True, text=True)
    first, *lines = out.stdout.split("\n")
    P, pages = 1 << shift, int(first)
    # a row's last `tokens` tokens, wherever they end in a page, lie in as many pages, and a row has no more
    assert pages == min((tokens + P - 2) // P + 1, max_pages)
    assert len(lines) > 5 or n * pages * layers * G < 5
    for line in filter(None, lines):
        task, seq, layer, page, g = map(int, line.split())
        assert 0 <= seq < n and 0 <= layer < layers and 0 <= page < pages and 0 <= g < G
        assert ((seq * layers + layer) * pages + page) * G + g == task


def test_the_kernel_and_its_launch_take_this_split():
    f = functions("sparse.cu")
    assert "BoundsTask of(task, most, p.nlayers, pg.G);" in f["k_page_bounds"] and "bounds_pages(" in f["k_page_bounds"]
    assert "bounds_pages(" in f["page_bounds_launch"]
